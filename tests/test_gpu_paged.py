"""Attention over a paged latent cache (palu_attn_paged, palu_attn_prefix) against the float64 oracle, which is given the
attended rows of every sequence, gathered, with their positions.

Tolerance, per output element: half a step of the output's type, relative, plus a share of the row's largest output.
 float16   2^-11 + 2^-14: keys, queries and probabilities enter as pairs (2^-21 relative each), angles are right to 2e-7
           absolute and every float32 sum to a few 2^-24, so a logit sum(|q k|)/sqrt(128) (at most 24 for these inputs) is
           right to 24 * 1e-6, and so are the probabilities, relative; the merged latents are again a pair.
 bfloat16  2^-8 + 2^-8: keys and queries are rounded once to float16 (half a step 2^-11 each), so a logit is off by at most
           2^-10 * 24 / 8 in the root mean square over 128 products, 2^-8.4 with all of them at their worst at once; the
           probabilities change by that, relative, and the outputs, sums of them with random signs, by less.
"""

import numpy as np
import pytest
import torch

import paper_2407_21118_amd as P
from oracle import palu_oracle as O
from workloads import synth

pytestmark = pytest.mark.gpu

from gpu_util import make_desc, say, torch_dtype  # noqa: E402

TOL = {"f16": (2.0 ** -11, 2.0 ** -14), "bf16": (2.0 ** -8, 2.0 ** -8)}


def uneven_layer(theta=10000.0, q_per_kv=1):
    """Groups of 3, 1 and 5 heads, every one with ranks of its own."""
    return synth.Layer(9, 128, [0, 3, 4, 9], [0, 96, 128, 384], [0, 64, 320, 480], theta, q_per_kv=q_per_kv)


LAYERS = {
    "4x128": lambda: synth.uniform_layer(8, 4, 128),
    "4x256": lambda: synth.uniform_layer(8, 4, 256),
    "1x64": lambda: synth.uniform_layer(5, 1, 64),
    "1x32": lambda: synth.uniform_layer(2, 1, 32),
    "2x160-96": lambda: synth.uniform_layer(4, 2, 160, 96),
    "4x128-384": lambda: synth.uniform_layer(4, 4, 128, 384),
    "8x512": lambda: synth.uniform_layer(8, 8, 512, 512),
    "1x288": lambda: synth.uniform_layer(2, 1, 288, 32),
    "3x384-64": lambda: synth.uniform_layer(3, 3, 384, 64),
    "uneven": uneven_layer,
    "uneven-gqa3": lambda: uneven_layer(q_per_kv=3),
    "gqa4": lambda: synth.uniform_layer(8, 4, 256, rope_theta=500000.0, q_per_kv=4),
    "gqa8-2x96": lambda: synth.uniform_layer(4, 2, 96, q_per_kv=8),
    "gqa20": lambda: synth.uniform_layer(2, 1, 64, q_per_kv=20),
    "gqa70": lambda: synth.uniform_layer(2, 2, 64, q_per_kv=70),
    "gqa16-512": lambda: synth.uniform_layer(4, 4, 512, 256, q_per_kv=16),
    "norope": lambda: synth.uniform_layer(8, 4, 128, rope_theta=0.0),
}


class Pool:
    """A page pool whose unattended rows and pages are NaN and whose page table names no page twice."""

    def __init__(self, layer, dtype, lens, page_rows, seed=0, prefix=0, max_len=None, q_scale=1.5, extra_pages=3):
        rng = np.random.default_rng(seed)
        self.layer, self.dtype, self.lens, self.prefix, self.page_rows = layer, dtype, list(lens), prefix, page_rows
        self.max_len = max(max(lens), prefix, 1) if max_len is None else max_len
        B = len(lens)
        per_seq = -(-self.max_len // page_rows)
        n_pages = B * per_seq + extra_pages
        self.table = rng.permutation(n_pages)[:B * per_seq].reshape(B, per_seq).astype(np.int32)
        draw = lambda *s: synth.round_to(rng.standard_normal(s), dtype)  # noqa: E731
        self.hk = np.full((n_pages, page_rows, layer.R_k), np.nan, np.float32)
        self.hv = np.full((n_pages, page_rows, layer.R_v), np.nan, np.float32)
        self.rows = [draw(L, layer.R_k + layer.R_v) for L in lens]            # every sequence's own rows ...
        self.shared = draw(prefix, layer.R_k + layer.R_v)                     # ... of which those of the prefix are sequence 0's
        self.q = synth.round_to(q_scale * rng.standard_normal((B, layer.n_q_heads, 128)), dtype)
        self.Bk, self.Bv = (synth.round_to(np.concatenate([
            rng.standard_normal((off[j + 1] - off[j]) * layer.group_size(j) * 128) / np.sqrt(off[j + 1] - off[j])
            for j in range(layer.n_groups)]), dtype) for off in (layer.k_rank_off, layer.v_rank_off))

    def seen(self, b, window, n_sink):
        t = np.arange(self.lens[b])
        return t if window == 0 else t[(t < n_sink) | (t >= self.lens[b] - window)]

    def latents(self, b, t):
        """Rows t of sequence b, [n, R_k + R_v]."""
        both = np.concatenate([self.shared, self.rows[b][self.prefix:]])
        return both[t]

    def put(self, window, n_sink):
        """Writes the attended rows, and those alone, where the page table says."""
        pr = self.page_rows
        for b, L in enumerate(self.lens):
            t = self.seen(b, window, n_sink)
            t = t[t >= self.prefix]
            at = self.table[b, t // pr], t % pr
            x = self.latents(b, t)
            self.hk[at], self.hv[at] = x[:, : self.layer.R_k], x[:, self.layer.R_k:]
        t = np.arange(self.prefix)
        at = self.table[0, t // pr], t % pr
        self.hk[at], self.hv[at] = self.shared[:, : self.layer.R_k], self.shared[:, self.layer.R_k:]

    def reference(self, window=0, n_sink=0, q_pos=None):
        ly = self.layer
        out = np.zeros((len(self.lens), ly.n_q_heads, 128))
        for b, L in enumerate(self.lens):
            t = self.seen(b, window, n_sink)
            if len(t) == 0:
                continue
            x = self.latents(b, t)[None]
            pos = np.array([L - 1 if q_pos is None else q_pos[b]])
            out[b] = O.attn_decode(self.q[b:b + 1], pos, x[..., : ly.R_k], x[..., ly.R_k:], self.Bk, self.Bv, ly.group_head_off,
                                   ly.k_rank_off, ly.v_rank_off, 128, ly.rope_theta, t.astype(np.int32), None, ly.q_per_kv)[0]
        return out

    def device(self):
        dt = torch_dtype(self.dtype)
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dt).cuda()  # noqa: E731
        d = dict(q=dev(self.q), hk=dev(self.hk), hv=dev(self.hv), Bk=dev(self.Bk), Bv=dev(self.Bv))
        d["page_table"] = torch.from_numpy(self.table).cuda()
        d["seq_lens"] = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        d["rope_table"] = P.palu_rope_table_init(self.layer.rope_theta, 128, self.max_len)
        d["rope_table_len"] = self.max_len
        return d

    def call(self, d, window=0, n_sink=0, q_pos=None, **kw):
        desc = make_desc(self.layer, self.dtype)
        if self.prefix:
            return P.palu_attn_prefix(desc, len(self.lens), self.prefix, self.max_len, q_pos=q_pos, **d, **kw)
        return P.palu_attn_paged(desc, len(self.lens), self.max_len, q_pos=q_pos, window=window, n_sink=n_sink, **d, **kw)


def hold(got, ref, dtype):
    got = got.double().cpu().numpy()
    rel, share = TOL[dtype]
    assert np.isfinite(got).all()
    room = rel * np.abs(ref) + share * np.abs(ref).max(-1, keepdims=True)
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
    say(f"[paged] {name} {dtype}")
    check(Pool(LAYERS[name](), dtype, [200, 0, 1, 333, 64], 16))
    check(Pool(LAYERS[name](), dtype, [200, 3, 130], 32, seed=1), window=70, n_sink=5)


@pytest.mark.parametrize("page_rows", [1, 16, 64, 512])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (1, 1), (17, 4), (64, 64), (100, 70), (63, 129), (1000, 300)])
def test_windows_sinks_and_lengths(page_rows, window, n_sink):
    lens = [0, 1, 2, 63, 64, 65, 127, 128, 129, 191, 200, 317, 700]
    say(f"[paged] pages of {page_rows}, window {window}, sinks {n_sink}")
    check(Pool(synth.uniform_layer(4, 4, 64), "f16", lens, page_rows, seed=window + n_sink), window, n_sink)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("name", list(LAYERS))
def test_prefix_layers(name, dtype):
    say(f"[prefix] {name} {dtype}")
    check(Pool(LAYERS[name](), dtype, [200, 0, 201, 333, 264], 16, prefix=200))
    check(Pool(LAYERS[name](), dtype, [70] * 7, 32, seed=2, prefix=70))


@pytest.mark.parametrize("batch", [1, 2, 15, 17, 33, 70, 130])
@pytest.mark.parametrize("prefix,tail", [(1, 0), (63, 2), (64, 64), (100, 1), (129, 200)])
def test_prefix_lengths_and_batches(batch, prefix, tail):
    lens = [prefix + (tail * (i + 1)) // batch for i in range(batch)]
    if batch > 3:
        lens[2], lens[3] = 0, max(1, prefix // 2)                    # an idle slot; a sequence that ends inside the prefix
    say(f"[prefix] batch {batch}, {prefix} + up to {tail}")
    check(Pool(synth.uniform_layer(4, 4, 64, 32), "f16", lens, 16, seed=batch, prefix=prefix, max_len=max(lens) + 5))


def test_long_sequences_in_many_splits():
    say("[paged] 1 x 20011 rows, window 9999")
    check(Pool(synth.uniform_layer(8, 4, 128), "f16", [20011], 64, seed=5))
    check(Pool(synth.uniform_layer(8, 4, 128), "bf16", [20011, 9000], 64, seed=6), window=9999, n_sink=100)
    say("[prefix] 3 sequences behind 15001 rows")
    check(Pool(synth.uniform_layer(8, 4, 128), "f16", [15300, 15002, 16001], 64, seed=7, prefix=15001))


def test_peaked_softmax():
    """Logits of +-60: the maximum moves from tile to tile, and almost all probabilities are zero.  A logit's error grows with
    it: 24 * 16 products' worth, so the share of the largest output is 16 times that of the other tests."""
    pool = Pool(synth.uniform_layer(4, 4, 128), "f16", [700, 64, 1], 16, seed=8, q_scale=24.0)
    pool.put(0, 0)
    got = pool.call(pool.device()).double().cpu().numpy()
    ref = pool.reference()
    assert (np.abs(got - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -10 * np.abs(ref).max(-1, keepdims=True)).all()


def test_query_positions_of_the_callers_own():
    pool = Pool(synth.uniform_layer(4, 2, 96), "f16", [130, 70, 9], 16, seed=9, max_len=400)
    pool.put(50, 3)
    for pos in ([0, 399, 65], [130, 69, 8]):
        out = pool.call(pool.device(), 50, 3, q_pos=torch.tensor(pos, dtype=torch.int32, device="cuda"))
        hold(out, pool.reference(50, 3, pos), "f16")


def test_page_table_entries_that_are_not_read_and_bad_ones():
    """Entries of pages without an attended row hold anything; an entry that is read and out of range is clamped, so that the
    call stays within the pool (its values are then another page's)."""
    pool = Pool(synth.uniform_layer(4, 4, 64), "f16", [300, 40, 0], 16, seed=10)
    pool.put(50, 4)
    keep = {0: [0] + list(range(250 // 16, 299 // 16 + 1)), 1: [0, 1, 2], 2: []}
    for b in range(3):
        for i in range(pool.table.shape[1]):
            if i not in keep[b]:
                pool.table[b, i] = [-1, 2 ** 31 - 1, -2 ** 31][i % 3]
    hold(pool.call(pool.device(), 50, 4), pool.reference(50, 4), "f16")
    last = pool.hk.shape[0] - 1
    good = pool.table.copy()
    pool.table[1, 1] = last + 12345
    d = pool.device()
    got = pool.call(d, 50, 4)
    pool.table[1, 1] = last
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(pool.call(pool.device(), 50, 4)))
    hold(got[0:1], pool.reference(50, 4)[0:1], "f16")
    pool.table = good


def test_pool_beyond_32_bit_offsets():
    """Pages at the end of a pool of 5 GB per side."""
    layer = synth.uniform_layer(32, 4, 256)
    small = Pool(layer, "f16", [130, 77], 64, seed=11)
    small.put(0, 0)
    d = small.device()
    n = 20000                                                        # pages of 64 rows of 4 KiB
    for side in ("hk", "hv"):
        big = torch.empty(n, 64, 2048, dtype=torch.float16, device="cuda")
        big[-small.hk.shape[0]:] = d[side]
        d[side] = big
    d["page_table"] = d["page_table"] + (n - small.hk.shape[0])
    hold(small.call(d), small.reference(), "f16")


def test_captured_and_replayed_with_changing_inputs_on_another_stream():
    """Two graphs that share no workspace, replayed in turn with eager calls of the same shapes between them."""
    pools = [Pool(synth.uniform_layer(8, 4, 128), "f16", [300, 150, 222], 16, seed=12, prefix=p) for p in (0, 130)]
    stream = torch.cuda.Stream()
    runs = []
    for pool in pools:
        pool.put(0, 0)
        d = pool.device()
        out = torch.empty_like(d["q"])
        torch.cuda.synchronize()
        desc = make_desc(pool.layer, "f16")
        need = (P.palu_attn_prefix_workspace_bytes(desc, 3, pool.prefix, pool.max_len) if pool.prefix
                else P.palu_attn_paged_workspace_bytes(desc, 3, pool.max_len))
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


def test_same_bits_every_time_and_queries_apart():
    """No result depends on timing, on what the workspace held, or on the other sequences of the batch."""
    pool = Pool(synth.uniform_layer(8, 4, 256), "bf16", [500, 500, 500, 500], 32, seed=13)
    pool.put(0, 0)
    d = pool.device()
    first = pool.call(d)
    for fill in (0, 255, 127):
        need = P.palu_attn_paged_workspace_bytes(make_desc(pool.layer, "bf16"), 4, pool.max_len)
        assert torch.equal(first, pool.call(d, workspace=torch.full((need,), fill, dtype=torch.uint8, device="cuda")))
    d["seq_lens"] = torch.tensor([500, 0, 17, 500], dtype=torch.int32, device="cuda")
    again = pool.call(d)
    assert torch.equal(first[0], again[0]) and torch.equal(first[3], again[3]) and not again[1].any()


def test_append_then_attend_then_share():
    """As a server uses them: a prompt is projected into the pages of one sequence, copies of its page table share it, every
    sequence appends tokens of its own, and both forms of attention agree with each other and with the oracle."""
    layer = synth.uniform_layer(8, 4, 128)
    desc = make_desc(layer, "f16")
    d_model, pr, B, prompt, steps = layer.n_heads * 128, 16, 3, 133, 3
    g = torch.Generator(device="cuda").manual_seed(14)
    rand = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).half()  # noqa: E731
    Ak, Av = rand(d_model, layer.R_k, scale=d_model ** -0.5), rand(d_model, layer.R_v, scale=d_model ** -0.5)
    Bk, Bv = rand(layer.b_elems("k"), scale=128 ** -0.5), rand(layer.b_elems("v"), scale=128 ** -0.5)
    pages = -(-(prompt + steps) // pr)
    shared = prompt // pr
    table = torch.empty(B, pages, dtype=torch.int32, device="cuda")
    table[:, :shared] = torch.arange(shared, dtype=torch.int32, device="cuda") + 2
    table[:, shared:] = (torch.arange(B * (pages - shared), dtype=torch.int32, device="cuda") + 2 + shared).view(B, -1).flip(0)
    n_pages = 2 + shared + B * (pages - shared)
    hk = torch.full((n_pages, pr, layer.R_k), float("nan"), dtype=torch.float16, device="cuda")
    hv = torch.full((n_pages, pr, layer.R_v), float("nan"), dtype=torch.float16, device="cuda")

    def rows_of(b, t):
        return (table[b, t // pr] * pr + t % pr).int()

    t = torch.arange(prompt, device="cuda")
    x = rand(prompt, d_model)
    P.palu_encode_kv(desc, x, Ak, Av, hk, layer.R_k, hv, layer.R_v, dst_row=rows_of(0, t))
    for b in range(1, B):                                            # the page that the prompt ends in is copied for the others
        hk[table[b, shared].long()] = hk[table[0, shared].long()]
        hv[table[b, shared].long()] = hv[table[0, shared].long()]
    rope = P.palu_rope_table_init(layer.rope_theta, 128, prompt + steps)
    for i in range(steps):
        x, q = rand(B, d_model), rand(B, 8, 128)
        at = torch.tensor([prompt + i], device="cuda")
        P.palu_encode_kv(desc, x, Ak, Av, hk, layer.R_k, hv, layer.R_v, dst_row=torch.cat([rows_of(b, at) for b in range(B)]))
        lens = torch.full((B,), prompt + i + 1, dtype=torch.int32, device="cuda")
        args = (q, None, hk, hv, table, lens, Bk, Bv, rope, prompt + steps)
        alone = P.palu_attn_paged(desc, B, prompt + steps, *args)
        joint = P.palu_attn_prefix(desc, B, prompt, prompt + steps, *args)
        late = P.palu_attn_paged(desc, B, prompt + steps, *args, window=40, n_sink=4)
        torch.cuda.synchronize()
        for b in range(B):
            L = prompt + i + 1
            at = rows_of(b, torch.arange(L, device="cuda")).long()
            HK, HV = (h.view(-1, h.shape[-1])[at].double().cpu().numpy()[None] for h in (hk, hv))
            pos = np.arange(L)
            for got, sel in ((alone, pos), (joint, pos), (late, pos[(pos < 4) | (pos >= L - 40)])):
                ref = O.attn_decode(q[b:b + 1].double().cpu().numpy(), np.array([L - 1]), HK[:, sel], HV[:, sel],
                                    Bk.double().cpu().numpy(), Bv.double().cpu().numpy(), layer.group_head_off, layer.k_rank_off,
                                    layer.v_rank_off, 128, layer.rope_theta, sel.astype(np.int32))
                hold(got[b:b + 1], ref, "f16")


@pytest.mark.parametrize("name,dtype", [("4x256", "f16"), ("gqa4", "bf16"), ("wide values", "f16"), ("wide keys", "bf16")])
def test_shared_and_own_rows_in_many_splits(name, dtype):
    """Sequences of very different lengths behind a prefix of many tiles: splits of both kinds, in one launch, by up to 64 query rows."""
    layer = {"wide values": lambda: synth.uniform_layer(8, 4, 256, 384), "wide keys": lambda: synth.uniform_layer(4, 2, 512, 256)}.get(name, LAYERS.get(name))()
    lens = [2500 + (137 * i * i) % 701 for i in range(18)] + [0, 1, 1300]
    say(f"[prefix] {name} {dtype}: 21 sequences behind 2500 rows")
    check(Pool(layer, dtype, lens, 32, seed=15, prefix=2500, max_len=3300))


def test_many_query_rows_over_a_window_with_sinks_far_apart():
    """The jump from the sinks to the window lies inside a workgroup's run of tiles, for 20 and 70 query rows per head."""
    for name in ("gqa20", "gqa70"):
        say(f"[paged] {name}, window 700 of 3000 rows")
        check(Pool(LAYERS[name](), "f16", [3000, 2999, 31, 740], 16, seed=16), window=700, n_sink=100)


def test_queries_of_one_sequence_as_entries_of_the_batch():
    """A speculative-decoding check: three entries with one page-table row and lengths of their own; as one by one."""
    pool = Pool(synth.uniform_layer(8, 4, 128), "f16", [400, 400, 400], 16, seed=17)
    pool.put(0, 0)
    d = pool.device()
    d["page_table"][1:] = d["page_table"][0]
    d["seq_lens"] = torch.tensor([400, 399, 398], dtype=torch.int32, device="cuda")
    got = pool.call(d, 90, 4)
    pool.rows[1], pool.rows[2], pool.lens = pool.rows[0], pool.rows[0], [400, 399, 398]
    hold(got, pool.reference(90, 4), "f16")


def test_lengths_left_out():
    """Without seq_lens every sequence has max_len rows, its query the position of the last."""
    for prefix in (0, 100):
        pool = Pool(synth.uniform_layer(8, 4, 128), "bf16", [260, 260], 16, seed=18, prefix=prefix)
        pool.put(0, 0)
        d = pool.device()
        d["seq_lens"] = None
        hold(pool.call(d), pool.reference(), "bf16")


def test_two_calls_at_once_on_two_streams():
    """Workspaces of their own; each as when it runs alone."""
    pools = [Pool(synth.uniform_layer(8, 4, 256), "f16", [2000, 1500, 1777], 64, seed=19 + p, prefix=p) for p in (0, 1400)]
    runs = []
    for pool in pools:
        pool.put(0, 0)
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
