"""Attention over a paged cache held in 4 bits (palu_attn_paged_quant) against the float64 oracle, which is given what the attended
rows of every sequence stand for, (code - zero) * scale in 64 bits, with their positions.

Tolerance, per output element: half a step of the output's type, relative (2^-11, bfloat16 2^-8), plus a share of the row's largest
output.  The share: codes are exact, the weights enter as they are (float16) or right to 2^-39 of the largest (bfloat16), angles are
right to 1e-6 and every float32 sum to a few 2^-24, so a logit sum(|q k|)/sqrt(128) (at most 24 for these inputs) is right to
24 * 2e-6 = 2^-14.3 in natural units, and so is every probability, relative; an output is a weighted mean whose weights' errors have either
sign.  2^-14 for float16; for bfloat16 the merged latents enter as a pair of bfloat16 numbers (2^-16 each, of 128 or more with either sign), 2^-13."""

import numpy as np
import pytest
import torch

import paper_2407_21118_amd as P
from oracle import palu_oracle as O
from workloads import synth

pytestmark = pytest.mark.gpu

from gpu_util import say, torch_dtype  # noqa: E402

TOL = {"f16": (2.0 ** -11, 2.0 ** -14), "bf16": (2.0 ** -8, 2.0 ** -13)}


def make_desc(layer, dtype, bits=P.PALU_I4):
    return P.LayerDesc(layer.n_heads, 128, layer.group_head_off, layer.k_rank_off, layer.v_rank_off,
                       P.PALU_F16 if dtype == "f16" else P.PALU_BF16, bits, bits, 128, layer.rope_theta, layer.q_per_kv)


def uneven_layer(theta=10000.0, q_per_kv=1):
    """Groups of 3, 1, 5 and 2 heads, every one with ranks of its own."""
    return synth.Layer(11, 128, [0, 3, 4, 9, 11], [0, 256, 384, 896, 1024], [0, 128, 384, 896, 1280], theta, q_per_kv=q_per_kv)


LAYERS = {
    "4x128": lambda: synth.uniform_layer(8, 4, 128),
    "4x256": lambda: synth.uniform_layer(8, 4, 256),
    "1x128": lambda: synth.uniform_layer(5, 1, 128),
    "2x128-256": lambda: synth.uniform_layer(6, 2, 128, 256),
    "2x256-128": lambda: synth.uniform_layer(4, 2, 256, 128),
    "4x128-384": lambda: synth.uniform_layer(4, 4, 128, 384),
    "8x512": lambda: synth.uniform_layer(8, 8, 512, 512),
    "5x384-256": lambda: synth.uniform_layer(10, 5, 384, 256),
    "1x256-512": lambda: synth.uniform_layer(3, 1, 256, 512),
    "uneven": uneven_layer,
    "uneven-gqa3": lambda: uneven_layer(q_per_kv=3),
    "gqa2": lambda: synth.uniform_layer(8, 4, 256, rope_theta=500000.0, q_per_kv=2),
    "gqa4": lambda: synth.uniform_layer(8, 4, 256, rope_theta=500000.0, q_per_kv=4),
    "gqa8-2x128": lambda: synth.uniform_layer(4, 2, 128, q_per_kv=8),
    "gqa4-256-384": lambda: synth.uniform_layer(8, 4, 256, 384, q_per_kv=4),
    "gqa2-128-512": lambda: synth.uniform_layer(5, 5, 128, 512, q_per_kv=2),
    "8x256-512": lambda: synth.uniform_layer(8, 8, 256, 512),
    "gqa20-512": lambda: synth.uniform_layer(4, 4, 512, q_per_kv=20),
    "gqa70": lambda: synth.uniform_layer(2, 2, 128, q_per_kv=70),
    "norope": lambda: synth.uniform_layer(8, 4, 128, rope_theta=0.0),
    "theta1000": lambda: synth.uniform_layer(8, 4, 256, rope_theta=1000.0),
    "theta30": lambda: synth.uniform_layer(4, 4, 128, rope_theta=30.0, q_per_kv=2),
}


class Pool:
    """A page pool whose unattended rows have NaN for scales and zero-points, and whose page table names no page twice.
    shape: how the rows' scales and zero-points are drawn; "normal": those of quantised normal latents."""

    def __init__(self, layer, dtype, lens, page_rows, seed=0, max_len=None, q_scale=1.5, extra_pages=3, shape="normal"):
        rng = np.random.default_rng(seed)
        self.layer, self.dtype, self.lens, self.page_rows = layer, dtype, list(lens), page_rows
        self.max_len = max(max(lens), 1) if max_len is None else max_len
        B = len(lens)
        per_seq = -(-self.max_len // page_rows)
        self.n_pages = B * per_seq + extra_pages
        self.table = rng.permutation(self.n_pages)[:B * per_seq].reshape(B, per_seq).astype(np.int32)
        self.rows, self.pool = {}, {}
        for side, R in (("k", layer.R_k), ("v", layer.R_v)):
            self.pool[side] = (np.full((self.n_pages, page_rows, R // 2), 0xA7, np.uint8),
                               np.full((self.n_pages, page_rows, R // 128), np.nan, np.float16),
                               np.full((self.n_pages, page_rows, R // 128), np.nan, np.float16))
            self.rows[side] = [self.draw(rng, L, R, shape, side) for L in lens]
        self.q = synth.round_to(q_scale * rng.standard_normal((B, layer.n_q_heads, 128)), dtype)
        self.Bk, self.Bv = (synth.round_to(np.concatenate([
            rng.standard_normal((off[j + 1] - off[j]) * layer.group_size(j) * 128) / np.sqrt(off[j + 1] - off[j])
            for j in range(layer.n_groups)]), dtype) for off in (layer.k_rank_off, layer.v_rank_off))

    @staticmethod
    def draw(rng, L, R, shape, side):
        packed, s, z = O.quant_latent(rng.standard_normal((L, R)).astype(np.float16)) if L else (
            np.zeros((0, R // 2), np.uint8), np.zeros((0, R // 128), np.float16), np.zeros((0, R // 128), np.float16))
        if shape == "far zeros":                               # a block far from zero: values 0.3 in size all the same
            far = rng.choice([0, 900, -1000, 2100, -5000, 30000], size=z.shape, p=[0.75, 0.05, 0.05, 0.05, 0.05, 0.05])
            s = np.where(far != 0, 0.3 / np.maximum(np.abs(far), 1), s).astype(np.float16)
            z = np.where(far != 0, far, z).astype(np.float16)
        elif shape == "odd zeros":                             # any float16 number is a zero-point
            z = (z + rng.uniform(-1, 1, z.shape)).astype(np.float16)
        elif shape == "scales":                                # of every size, none and below none
            s = (s * 10.0 ** rng.uniform(-5.5, 0, s.shape) * rng.choice([1, 1, 1, -1, 0], size=s.shape)).astype(np.float16)
        return packed, s, z

    def seen(self, b, window, n_sink):
        t = np.arange(self.lens[b])
        return t if window == 0 else t[(t < n_sink) | (t >= self.lens[b] - window)]

    def put(self, window=0, n_sink=0):
        """Writes the attended rows, and those alone, where the page table says."""
        for b in range(len(self.lens)):
            t = self.seen(b, window, n_sink)
            at = self.table[b, t // self.page_rows], t % self.page_rows
            for side in "kv":
                for x, y in zip(self.pool[side], self.rows[side][b]):
                    x[at] = y[t]

    def reference(self, window=0, n_sink=0, q_pos=None):
        ly = self.layer
        out = np.zeros((len(self.lens), ly.n_q_heads, 128))
        for b, L in enumerate(self.lens):
            t = self.seen(b, window, n_sink)
            if len(t) == 0:
                continue
            hk, hv = (O.dequant_latent(*(y[t] for y in self.rows[side][b]))[None] for side in "kv")
            pos = np.array([L - 1 if q_pos is None else q_pos[b]])
            out[b] = O.attn_decode(self.q[b:b + 1], pos, hk, hv, self.Bk, self.Bv, ly.group_head_off, ly.k_rank_off, ly.v_rank_off, 128,
                                   ly.rope_theta, t.astype(np.int32), None, ly.q_per_kv)[0]
        return out

    def device(self):
        dt = torch_dtype(self.dtype)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dt).cuda()  # noqa: E731
        d = dict(q=dev(self.q), Bk=dev(self.Bk), Bv=dev(self.Bv))
        for side in "kv":
            d["h" + side], d[f"h{side}_scale"], d[f"h{side}_zero"] = (torch.from_numpy(x.copy()).cuda() for x in self.pool[side])
        d["page_table"] = torch.from_numpy(self.table).cuda()
        d["seq_lens"] = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        d["rope_table"] = P.palu_rope_table_init(self.layer.rope_theta, 128, self.max_len)
        d["rope_table_len"] = self.max_len
        return d

    def call(self, d, window=0, n_sink=0, q_pos=None, **kw):
        return P.palu_attn_paged_quant(make_desc(self.layer, self.dtype), len(self.lens), self.max_len, q_pos=q_pos, window=window,
                                       n_sink=n_sink, **d, **kw)


def hold(got, ref, dtype, share=None):
    got = got.double().cpu().numpy()
    rel, usual = TOL[dtype]
    assert np.isfinite(got).all()
    room = rel * np.abs(ref) + (usual if share is None else share) * np.abs(ref).max(-1, keepdims=True)
    off = np.abs(got - ref)
    worst = float((off / np.maximum(room, 1e-30)).max())
    say(f"    worst element at {worst:.3f} of its tolerance")
    assert (off <= room).all(), worst


def check(pool, window=0, n_sink=0):
    pool.put(window, n_sink)
    d = pool.device()
    out = torch.full((len(pool.lens), pool.layer.n_q_heads, 128), float("nan"), dtype=d["q"].dtype, device="cuda")
    pool.call(d, window, n_sink, out=out)
    torch.cuda.synchronize()
    hold(out, pool.reference(window, n_sink), pool.dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("name", list(LAYERS))
def test_layers_all_rows_and_a_window(name, dtype):
    say(f"[paged 4 bits] {name} {dtype}")
    check(Pool(LAYERS[name](), dtype, [200, 0, 1, 333, 64], 16))
    check(Pool(LAYERS[name](), dtype, [200, 3, 130], 32, seed=1), window=70, n_sink=5)


@pytest.mark.parametrize("page_rows", [1, 16, 64, 512])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (1, 1), (17, 4), (64, 64), (100, 70), (63, 129), (1000, 300)])
def test_windows_sinks_and_lengths(page_rows, window, n_sink):
    lens = [0, 1, 2, 63, 64, 65, 127, 128, 129, 191, 200, 317, 700]
    say(f"[paged 4 bits] pages of {page_rows}, window {window}, sinks {n_sink}")
    check(Pool(synth.uniform_layer(4, 4, 128), "f16", lens, page_rows, seed=window + n_sink), window, n_sink)


@pytest.mark.parametrize("shape", ["far zeros", "odd zeros", "scales"])
@pytest.mark.parametrize("name,dtype", [("4x256", "f16"), ("4x128-384", "bf16"), ("gqa4", "f16"), ("8x512", "bf16")])
def test_scales_and_zero_points_of_any_size(name, dtype, shape):
    say(f"[paged 4 bits] {name} {dtype}, {shape}")
    check(Pool(LAYERS[name](), dtype, [200, 517, 33, 300], 16, seed=3, shape=shape))
    check(Pool(LAYERS[name](), dtype, [700], 16, seed=4, shape=shape), window=301, n_sink=40)


def test_long_sequences_in_many_splits():
    say("[paged 4 bits] 1 x 20011 rows, window 9999")
    check(Pool(synth.uniform_layer(8, 4, 128), "f16", [20011], 64, seed=5))
    check(Pool(synth.uniform_layer(8, 4, 256), "bf16", [20011, 9000], 64, seed=6), window=9999, n_sink=100)


@pytest.mark.parametrize("name", ["4x256", "gqa4", "gqa20-512"])
def test_peaked_softmax(name):
    """Logits of +-60: the maximum moves along the sequence, and almost all probabilities are zero.  A logit's error grows with
    it: 24 * 16 products' worth, so the share of the largest output is 16 times that of the other tests."""
    pool = Pool(LAYERS[name](), "f16", [700, 64, 1], 16, seed=8, q_scale=24.0)
    pool.put()
    hold(pool.call(pool.device()), pool.reference(), "f16", share=2.0 ** -10)


def test_query_positions_of_the_callers_own():
    pool = Pool(synth.uniform_layer(4, 2, 128), "f16", [130, 70, 9], 16, seed=9, max_len=400)
    pool.put(50, 3)
    for pos in ([0, 399, 65], [130, 69, 8]):
        out = pool.call(pool.device(), 50, 3, q_pos=torch.tensor(pos, dtype=torch.int32, device="cuda"))
        hold(out, pool.reference(50, 3, pos), "f16")


def test_page_table_entries_that_are_not_read_and_bad_ones():
    """Entries of pages without an attended row hold anything; an entry that is read and out of range is clamped, so that the
    call stays within the pool (its values are then another page's)."""
    pool = Pool(synth.uniform_layer(4, 4, 128), "f16", [300, 40, 0], 16, seed=10)
    pool.put(50, 4)
    keep = {0: [0] + list(range(250 // 16, 299 // 16 + 1)), 1: [0, 1, 2], 2: []}
    for b in range(3):
        for i in range(pool.table.shape[1]):
            if i not in keep[b]:
                pool.table[b, i] = [-1, 2 ** 31 - 1, -2 ** 31][i % 3]
    hold(pool.call(pool.device(), 50, 4), pool.reference(50, 4), "f16")
    last = pool.n_pages - 1
    pool.table[1, 1] = last + 12345
    got = pool.call(pool.device(), 50, 4)
    pool.table[1, 1] = last
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(pool.call(pool.device(), 50, 4)))
    hold(got[0:1], pool.reference(50, 4)[0:1], "f16")


def test_lengths_out_of_range_and_left_out():
    """Lengths are clamped to [0, max_len]; without them every sequence has max_len rows, its query the position of the last."""
    pool = Pool(synth.uniform_layer(8, 4, 128), "bf16", [260, 260, 260], 16, seed=18)
    pool.put()
    d = pool.device()
    d["seq_lens"] = torch.tensor([260, 2 ** 31 - 1, -7], dtype=torch.int32, device="cuda")
    got = pool.call(d)
    assert not got[2].any()
    hold(got[:2], pool.reference()[:2], "bf16")
    d["seq_lens"] = None
    hold(pool.call(d), pool.reference(), "bf16")


def test_not_a_number_stays_in_its_heads():
    """NaN in a query makes that head's output NaN; in an attended row's scale or zero-point all heads of its group, and no others."""
    pool = Pool(synth.uniform_layer(8, 4, 128), "f16", [150, 90], 16, seed=20)
    pool.put()
    ref = pool.reference()
    d = pool.device()
    d["q"][0, 3, 17] = float("nan")
    got = pool.call(d).cpu()
    assert got[0, 3].isnan().all()
    got[0, 3] = torch.from_numpy(ref[0, 3])
    hold(got, ref, "f16")
    for name in ("hk_scale", "hk_zero", "hv_scale", "hv_zero"):
        d = pool.device()
        d[name][int(pool.table[1, 2]), 7, 1] = float("nan")          # row 39 of sequence 1, the second group's
        got = pool.call(d).cpu()
        assert got[1, 4:].isnan().all(), name
        got[1, 4:] = torch.from_numpy(ref[1, 4:])
        hold(got, ref, "f16")


def test_pool_beyond_32_bit_offsets():
    """Pages at the end of a pool of 5 GB of codes per side."""
    layer = synth.uniform_layer(32, 4, 256)
    small = Pool(layer, "f16", [130, 77], 64, seed=11)
    small.put()
    d = small.device()
    n = 80000                                                        # pages of 64 rows of 1 KiB
    for name in ("hk", "hv", "hk_scale", "hk_zero", "hv_scale", "hv_zero"):
        big = torch.empty(n, 64, d[name].shape[2], dtype=d[name].dtype, device="cuda")
        big[-small.n_pages:] = d[name]
        d[name] = big
    d["page_table"] = d["page_table"] + (n - small.n_pages)
    hold(small.call(d), small.reference(), "f16")


def test_captured_and_replayed_with_changing_inputs_on_another_stream():
    """Two graphs that share no workspace, replayed in turn with eager calls of the same shapes between them."""
    pools = [Pool(LAYERS[name](), "f16", [300, 150, 222], 16, seed=12) for name in ("4x256", "gqa4")]
    stream = torch.cuda.Stream()
    runs = []
    for pool in pools:
        pool.put()
        d = pool.device()
        out = torch.empty_like(d["q"])
        torch.cuda.synchronize()
        need = P.palu_attn_paged_quant_workspace_bytes(make_desc(pool.layer, "f16"), 3, pool.max_len)
        work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")      # NaN everywhere
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            pool.call(d, out=out, workspace=work)
        runs.append((pool, d, out, graph))
    for k in range(4):
        for pool, d, out, graph in runs:
            d["q"].copy_(torch.randn(d["q"].shape, generator=torch.Generator().manual_seed(k)).to(torch.float16))
            d["seq_lens"].copy_(torch.tensor([300 - 7 * k, 150 - k, 0 if k == 2 else 222], dtype=torch.int32))
            out.fill_(float("nan"))
            graph.replay()
            eager = pool.call(d)
            torch.cuda.synchronize()
            assert torch.equal(out, eager)


def test_same_bits_every_time_and_sequences_apart():
    """No result depends on timing, on what the workspace held, or on the other sequences of the batch."""
    pool = Pool(synth.uniform_layer(8, 4, 256), "bf16", [500, 500, 500, 500], 32, seed=13)
    pool.put()
    d = pool.device()
    first = pool.call(d)
    for fill in (0, 255, 127):
        need = P.palu_attn_paged_quant_workspace_bytes(make_desc(pool.layer, "bf16"), 4, pool.max_len)
        assert torch.equal(first, pool.call(d, workspace=torch.full((need,), fill, dtype=torch.uint8, device="cuda")))
    d["seq_lens"] = torch.tensor([500, 0, 17, 500], dtype=torch.int32, device="cuda")
    again = pool.call(d)
    assert torch.equal(first[0], again[0]) and torch.equal(first[3], again[3]) and not again[1].any()


@pytest.mark.parametrize("name", ["4x256", "gqa2", "8x512", "4x128-384", "gqa2-128-512"])
def test_short_sequences_and_angle_tables_no_longer_than_they(name):
    for seed, lens in enumerate(([1], [3], [16], [17], [33, 1], [64, 65, 2])):
        say(f"[paged 4 bits] {name}, {lens} rows")
        check(Pool(LAYERS[name](), "f16", lens, 16, seed=seed))


def test_many_query_rows_over_a_window_with_sinks_far_apart():
    """The jump from the sinks to the window lies inside a workgroup's run of tiles."""
    for name in ("4x256", "gqa4", "gqa20-512", "gqa70"):
        say(f"[paged 4 bits] {name}, window 700 of 3000 rows")
        check(Pool(LAYERS[name](), "f16", [3000, 2999, 31, 740], 16, seed=16), window=700, n_sink=100)


def test_queries_of_one_sequence_as_entries_of_the_batch():
    """A speculative-decoding check: three entries with one page-table row and lengths of their own; as one by one."""
    pool = Pool(synth.uniform_layer(8, 4, 128), "f16", [400, 400, 400], 16, seed=17)
    pool.put()
    d = pool.device()
    d["page_table"][1:] = d["page_table"][0]
    d["seq_lens"] = torch.tensor([400, 399, 398], dtype=torch.int32, device="cuda")
    got = pool.call(d, 90, 4)
    for side in "kv":
        pool.rows[side] = [tuple(x[:n] for x in pool.rows[side][0]) for n in (400, 399, 398)]
    pool.lens = [400, 399, 398]
    hold(got, pool.reference(90, 4), "f16")


def test_two_calls_at_once_on_two_streams():
    """Workspaces of their own; each as when it runs alone."""
    runs = []
    for seed, name in enumerate(("4x256", "gqa4")):
        pool = Pool(LAYERS[name](), "f16", [2000, 1500, 1777], 64, seed=19 + seed)
        pool.put()
        d = pool.device()
        runs.append((pool, d, pool.call(d), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for k in range(3):
        for pool, d, alone, stream in runs:
            with torch.cuda.stream(stream):
                got.append((alone, pool.call(d)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in got)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("name", ["4x128", "4x256", "4x128-384", "gqa4", "8x512"])
def test_small_values_beside_large_ones_that_cancel(name, dtype):
    """Equal scores; of 40 rows two have values of 15 and -15 times a scale, one has 7 of a scale 2^-17 as large, the others none.  The weights of
    the large two are equal, so that their rounding cancels; what is left are float32 sums of three products, of at most 8 weights each, and of three
    zero-points' shares, at most 8 weights each: four additions, off by 2^-23 of 15 weights each where bits are cut off, 2^-17 of a weight.
    (The output, 1.3e-6, is among the float16 numbers that are 2^-24 apart.)"""
    layer = LAYERS[name]()
    for first in ((0, 1, 2), (3, 39, 17), (30, 12, 38)):
        pool = Pool(layer, dtype, [40], 16, seed=21)
        pool.q[:] = 0
        packed, s, z = (x.copy() for x in pool.rows["v"][0])
        packed[:], s[:], z[:] = 0x88, 1.0, 8.0
        a, b, c = first
        packed[a], z[a] = 0xFF, 0.0
        packed[b], z[b] = 0x00, 15.0
        packed[c], s[c] = 0xFF, 2.0 ** -17
        pool.rows["v"][0] = (packed, s, z)
        for j in range(layer.n_groups):                        # output f is latent channel f of its group's values
            n, rv = layer.group_size(j), layer.v_rank_off[j + 1] - layer.v_rank_off[j]
            at = sum(layer.group_size(i) * 128 * (layer.v_rank_off[i + 1] - layer.v_rank_off[i]) for i in range(j))
            one = np.zeros((rv, n, 128), np.float32)
            one[np.arange(128), :, np.arange(128)] = 1.0
            pool.Bv[at:at + one.size] = one.reshape(-1)
        pool.put()
        got, want = pool.call(pool.device()).double().cpu().numpy(), 7 * 2.0 ** -17 / 40
        room = (2.0 ** -17 + TOL[dtype][0] * 7 * 2.0 ** -17) / 40 + (2.0 ** -25 if dtype == "f16" else 0.0)
        off = np.abs(got - want).max()
        say(f"[paged 4 bits] {name} {dtype}: off by {off / want:.4f} of it, tolerance {room / want:.4f}")
        assert off <= room


def test_error_of_a_long_sequence_beside_that_of_rounding():
    """65536 rows.  With E the distance of the output from 64 bits and R that of the rounded 64-bit output, relative 2-norms, E^2 - R^2 is the square of
    what the arithmetic adds.  Logits: 64 pairs, each right to 2e-6 of |q||k|, 3 on average, with either sign, over sqrt(128): 4.2e-6.
    Weights and values: pairs of 2^-22, sums of float32: as much again at most.  Together below 2^-17; 2^-16 for an estimate from 2048 outputs."""
    pool = Pool(synth.uniform_layer(16, 4, 128), "f16", [65536], 64, seed=22)
    pool.put()
    ref = pool.reference()
    got = pool.call(pool.device()).double().cpu().numpy()
    size = np.linalg.norm(ref)
    E, R = np.linalg.norm(got - ref) / size, np.linalg.norm(ref.astype(np.float16).astype(np.float64) - ref) / size
    more = np.sqrt(max(0.0, E ** 2 - R ** 2))
    say(f"[paged 4 bits] 1 x 65536 rows: {E:.3e} from 64 bits, rounding {R:.3e}, the arithmetic adds {more:.2e}")
    assert more <= 2.0 ** -16


@pytest.mark.parametrize("name", ["4x128", "gqa4", "8x512"])
@pytest.mark.parametrize("size,rows", [(2.0 ** -12, 5000), (2.0 ** 14, 700), (6e4, 60)])
def test_values_of_any_size(name, size, rows):
    """Latents far from 1 beside weights that make up for it: their mean may lie among the float16 numbers that are 2^-24 apart, a row's values (65520
    where 65504 was quantised beside zeros) beyond the largest.  The tolerance is the other tests', relative to the outputs."""
    pool = Pool(LAYERS[name](), "f16", [rows, 7, 33], 16, seed=23)
    rng = np.random.default_rng(24)
    for b, n in enumerate(pool.lens):
        h = np.clip(size * rng.standard_normal((n, pool.layer.R_v)), -65504.0, 65504.0)
        if size > 5e4:
            h = np.where(rng.random(h.shape) < 0.5, 65504.0, 0.0)
        pool.rows["v"][b] = O.quant_latent(h.astype(np.float16))
    if size < 1:
        pool.q *= 0.05                                         # means over many rows
    pool.Bv = synth.round_to(pool.Bv * 2.0 ** -np.round(np.log2(size)), "f16")
    pool.put()
    hold(pool.call(pool.device()), pool.reference(), "f16")


@pytest.mark.parametrize("name,dtype", [("gqa2", "f16"), ("gqa4", "bf16"), ("gqa20-512", "f16"), ("uneven-gqa3", "bf16"), ("theta30", "f16"), ("gqa70", "f16"),
                                        ("1x128", "f16"), ("2x128-256", "bf16"), ("8x512", "f16")])
def test_numbers_that_are_not_finite_stay_in_their_heads(name, dtype):
    """A query's NaN or infinity makes its own head's outputs NaN, also where every score is -infinity; one in an attended row's scale or zero-point
    those of all heads of its group.  All others are as without it."""
    layer = LAYERS[name]()
    pool = Pool(layer, dtype, [70, 1, 90], 16, seed=25)
    pool.put()
    ref, qk = pool.reference(), layer.q_per_kv

    def one(d, b, heads, what):
        got = pool.call(d).cpu()
        assert got[b, heads].isnan().all(), what
        got[b, heads] = torch.from_numpy(ref[b, heads]).to(got.dtype)
        hold(got, ref, dtype)

    for b, head, feature, value in ((0, 0, 3, "nan"), (1, 1, 40, "nan"), (2, layer.n_q_heads - 1, 100, "inf"), (1, 0, 5, "inf"), (1, 0, 5, "-inf"),
                                    (1, layer.n_q_heads // 2, 70, "inf"), (1, layer.n_q_heads // 2, 70, "-inf")):
        say(f"[paged 4 bits] {name} {dtype}: {value} in feature {feature} of query {head} of sequence {b}")
        d = pool.device()
        d["q"][b, head, feature] = float(value)
        one(d, b, [head], "query")
    for side, off in (("k", layer.k_rank_off), ("v", layer.v_rank_off)):
        for j in sorted({0, layer.n_groups - 1}):
            heads = list(range(layer.group_head_off[j] * qk, layer.group_head_off[j + 1] * qk))
            for b, t, value in ((2, 17, "nan"), (2, 17, "inf"), (1, 0, "inf"), (1, 0, "-inf")):
                for what in ("scale", "zero"):
                    for block in sorted({off[j] // 128, off[j + 1] // 128 - 1}):
                        d = pool.device()
                        d[f"h{side}_{what}"][int(pool.table[b, t // 16]), t % 16, block] = float(value)
                        one(d, b, heads, f"{side} {what} {value}, group {j}, block {block}")
