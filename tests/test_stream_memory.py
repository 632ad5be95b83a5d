"""Memory that the binding allocates for a call on a stream of the caller's choice: scratch and outputs come from that stream's memory, where
nothing else runs that may still use them, and outputs are marked as used by the current stream too.  No device: the library, the streams
and the device checks are stand-ins, allocations are the host's."""

import contextlib

import pytest
import torch

import paper_2407_21118_amd as P
from paper_2407_21118_amd import binding

F16, I32, U8 = torch.float16, torch.int32, torch.uint8


class Stream:
    cuda_stream = 0
    device = torch.device("cpu")


class Library:
    def __getattr__(self, name):
        return lambda *a: 0


@pytest.fixture
def log(monkeypatch):
    """(allocated tensors with the stream that was current, tensors that were marked for a stream)"""
    here = Stream()
    now, made, marked = [here], [], []
    empty = torch.empty

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def allocate(*a, **kw):
        t = empty(*a, **{**kw, "device": "cpu"})
        made.append((t, now[-1]))
        return t

    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "_need_cuda", lambda *t: None)
    monkeypatch.setattr(binding, "_here", lambda stream: (0, 0))
    monkeypatch.setattr(binding, "_addresses", lambda here, *t, strided=(): [0] * (len(t) + len(strided)))
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: marked.append((t, stream)))
    return here, made, marked


def z(*shape, dtype=F16):
    return torch.zeros(shape, dtype=dtype)


def layer(**kw):
    return P.LayerDesc(2, 128, [0, 2], [0, 128], [0, 128], **kw)


PAGES = (z(2, 2, 128), None, z(3, 16, 128), z(3, 16, 128), z(2, 1, dtype=I32), None, z(128 * 256), z(128 * 256), z(0, dtype=U8), 0)
DENSE = (z(2, 2, 128), None, z(2, 16, 128), z(2, 16, 128), z(128 * 256), z(128 * 256), z(0), 0)
QUANT = (z(2, 2, 128), None, *[x for _ in "kv" for x in (z(3, 16, 64, dtype=U8), z(3, 16, 1), z(3, 16, 1))], z(2, 1, dtype=I32), None,
         z(128 * 256), z(128 * 256), z(0, dtype=U8), 0)
# (call, tensors that it hands to the caller)
CALLS = {
    "rope table": (lambda **kw: P.palu_rope_table_init(1e4, 128, 4, **kw), 1),
    "encode": (lambda **kw: P.palu_encode(layer(), 0, z(4, 256), z(256, 128), z(4, 128), 128, **kw), 0),
    "encode both": (lambda **kw: P.palu_encode_kv(layer(), z(4, 256), z(256, 128), z(256, 128), z(4, 128), 128, z(4, 128), 128, **kw), 0),
    "decode": (lambda **kw: P.palu_attn_decode(layer(), 2, 16, 16, *DENSE, **kw), 1),
    "decode, latent": (lambda **kw: P.palu_attn_decode_latent(layer(), 2, 16, 16, *DENSE[:5], *DENSE[6:], **kw), 1),
    "decode, several": (lambda **kw: P.palu_attn_decode_multi(layer(), 2, 3, 16, 16, *DENSE, **kw), 1),
    "step": (lambda **kw: P.palu_decode_step(layer(), 2, 16, 16, z(2, 256), z(0), z(0), None, *DENSE, **kw), 1),
    "step, transposed": (lambda **kw: P.palu_decode_step_t(layer(), 2, 16, 16, z(2, 256), z(0), z(0), None, *DENSE, **kw), 1),
    "paged": (lambda **kw: P.palu_attn_paged(layer(), 2, 16, *PAGES, **kw), 1),
    "prefix": (lambda **kw: P.palu_attn_prefix(layer(), 2, 8, 16, *PAGES, **kw), 1),
    "paged 4 bits": (lambda **kw: P.palu_attn_paged_quant(layer(k_latent_dtype=P.PALU_I4, v_latent_dtype=P.PALU_I4), 2, 16, *QUANT, **kw), 1),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_on_a_stream_of_its_own(log, name):
    here, made, marked = log
    call, kept = CALLS[name]
    other = Stream()
    got = call(stream=other)
    assert made and all(stream is other for _, stream in made)
    assert len(marked) == kept and all(t is got and stream is here for t, stream in marked)


@pytest.mark.parametrize("name", list(CALLS))
def test_on_the_current_stream(log, name):
    here, made, marked = log
    for stream in (None, here):
        CALLS[name][0](stream=stream)
    assert made and all(s is here for _, s in made) and not marked


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["decode", "paged", "paged 4 bits"])
def test_busy_streams(name):
    """The call's stream is busy when the call returns, and the current stream allocates and writes memory of the scratch's size; the current stream is
    busy when the call is made, and what it still reads has been freed."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(F16)  # noqa: E731
    B, L, rows = 3, 400, 416
    d = dict(n_heads=8, d_head=128, group_head_off=[0, 4, 8], k_rank_off=[0, 128, 256], v_rank_off=[0, 128, 256])
    table = P.palu_rope_table_init(1e4, 128, rows)
    q, Bk, Bv, pages = rand(B, 8, 128), rand(128 * 1024) * 0.1, rand(128 * 1024) * 0.1, torch.arange(B * 26, dtype=I32, device="cuda").view(B, 26)
    hk, hv = rand(B * 26, 16, 256), rand(B * 26, 16, 256)
    if name == "decode":
        desc, need = P.LayerDesc(**d), P.palu_attn_decode_workspace_bytes(P.LayerDesc(**d), B, rows)
        pos = torch.full((B,), L - 1, dtype=I32, device="cuda")
        call = lambda **kw: P.palu_attn_decode(desc, B, L, rows, q, pos, hk.view(B, rows, 256), hv.view(B, rows, 256), Bk, Bv, table, rows, **kw)  # noqa: E731
    elif name == "paged":
        desc, need = P.LayerDesc(**d), P.palu_attn_paged_workspace_bytes(P.LayerDesc(**d), B, L)
        call = lambda **kw: P.palu_attn_paged(desc, B, L, q, None, hk, hv, pages, None, Bk, Bv, table, rows, **kw)  # noqa: E731
    else:
        desc = P.LayerDesc(**d, k_latent_dtype=P.PALU_I4, v_latent_dtype=P.PALU_I4)
        need = P.palu_attn_paged_quant_workspace_bytes(desc, B, L)
        held = [torch.empty(B * 26, 16, w, dtype=t, device="cuda") for _ in "kv" for w, t in ((128, U8), (2, F16), (2, F16))]
        P.palu_quant_latent_kv(desc, hk.view(-1, 256), hv.view(-1, 256), *held)
        call = lambda **kw: P.palu_attn_paged_quant(desc, B, L, q, None, *held, pages, None, Bk, Bv, table, rows, **kw)  # noqa: E731
    alone = call()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    busy, mine = torch.zeros(1 << 26, device="cuda"), torch.zeros(1 << 26, device="cuda")
    for _ in range(3):
        with torch.cuda.stream(stream):
            for _ in range(20):
                busy.add_(1.0)
        got = call(stream=stream)
        after = [torch.empty(need, dtype=U8, device="cuda").fill_(255) for _ in range(8)]
        after += [torch.full_like(alone, float("nan")) for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(got, alone)
        del after, got
        before = [torch.empty(need, dtype=U8, device="cuda").fill_(7) for _ in range(8)]
        torch.cuda.synchronize()
        for _ in range(20):
            mine.add_(1.0)
        copies = [x.clone() for x in before]
        del before
        got = call(stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, alone) and all((x == 7).all() for x in copies)
        del copies, got
