"""Attention of single new tokens over a paged low-rank latent KV-cache: timed cases and the operators' definition.

Two operators on one compressed attention layer, whose key/value heads come in groups of `group` heads with latents of
`rk` (keys) and `rv` (values) channels per group, `q_per_kv` query heads to a key/value head:

  window   every sequence attends its first `sinks` rows and its newest `window` rows (window 0: all rows)
  prefix   the sequences of the batch share their first `prefix` rows, which are stored once; every sequence attends
           those and its own rows behind them

Row t of a sequence is row t % page of page page_table[b, t // page] of the caches, and its position is t.  With
K[t] = H_k[t] B_k (per key/value head), rotated to position t, and the query rotated to its own position,
  out = softmax_t(q . K[t] / sqrt(128)) H_v[t] B_v    over the attended rows, zeros where there are none.
"""

import math

import numpy as np
import torch

own = False
D = 128


def _case(name, op, heads=32, group=4, rk=256, rv=256, q_per_kv=1, theta=10000.0, dtype="f16", batch=1, length=1,
          ragged=False, page=64, window=0, sinks=0, prefix=0):
    """heads: key/value heads; length: rows of the longest sequence; ragged: the others are shorter, one slot is idle."""
    c = dict(op=op, heads=heads, group=group, rk=rk, rv=rv, q_per_kv=q_per_kv, theta=theta, dtype=dtype, batch=batch,
             length=length, ragged=ragged, page=page, window=window, sinks=sinks, prefix=prefix)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: a short chat turn on a small layer; launches and host time are what it costs
        _case("window-small-1x333", "window", heads=8, rk=128, rv=128, length=333, page=16, window=200, sinks=4),
        # one long stream on a 7B-shaped layer: the cache has grown to 16K rows, 4K of them are still seen
        _case("window-1x16k-w4096", "window", length=16384, window=4096, sinks=4),
        # a serving batch of streams of different lengths, bfloat16
        _case("window-24x8k-w1024-bf16", "window", dtype="bf16", batch=24, length=8190, ragged=True, page=16, window=1024, sinks=64),
        # grouped-query model without a window: four query heads share each key/value head
        _case("paged-gqa-4x16k", "window", heads=8, q_per_kv=4, theta=500000.0, batch=4, length=16384),
        # one latent per head, low rank, sequences of different lengths
        _case("paged-per-head-8x16k-bf16", "window", group=1, rk=64, rv=64, dtype="bf16", batch=8, length=16384, ragged=True, page=32),
        # keys compressed by 75 %, values by 25 %
        _case("window-4x16k-k128-v384", "window", rk=128, rv=384, batch=4, length=16000, ragged=True, window=6000, sinks=128),
        # the largest of these: a serving batch that sees everything
        _case("paged-16x8k", "window", batch=16, length=8192),
        # a few samples of one short prompt on a small layer
        _case("prefix-small-3x120", "prefix", heads=8, rk=128, rv=128, batch=3, length=150, ragged=True, page=16, prefix=111),
        # samples of one long document
        _case("prefix-8x16k", "prefix", batch=8, length=16384 + 256, ragged=True, prefix=16384),
        # a system prompt in front of a serving batch, bfloat16
        _case("prefix-64x4k-bf16", "prefix", dtype="bf16", batch=64, length=4096 + 700, ragged=True, page=16, prefix=4096),
        # the same on a grouped-query model
        _case("prefix-gqa-48x8k", "prefix", heads=8, q_per_kv=4, theta=500000.0, batch=48, length=8192 + 333, ragged=True, prefix=8192),
        # one latent per head, low rank, a long shared document
        _case("prefix-per-head-32x32k", "prefix", group=1, rk=64, rv=64, batch=32, length=32768 + 100, page=32, prefix=32768),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi], odd ones among them."""
    return int(round(lo * (hi / lo) ** rng.random()))


# what one drawn case may ask for: no more than the largest listed one
_MAX_FLOPS = 2.8e11
_MAX_BYTES = 1.0e9


def draw(rng):
    op = rng.choice(["window", "prefix"])
    heads, group, q_per_kv = rng.choice([(8, 4, 1), (32, 1, 1), (32, 2, 1), (32, 4, 1), (32, 4, 1), (8, 4, 4), (8, 2, 4), (4, 4, 8), (16, 8, 1)])
    rk, rv = (min(512, rng.choice([32, 64, 64, 96]) * group) for _ in range(2))
    dtype, theta = rng.choice(["f16", "bf16"]), rng.choice([10000.0, 500000.0])
    page, ragged = rng.choice([16, 32, 64, 128]), rng.random() < 0.7
    if op == "window":
        batch, length = _log_int(rng, 1, 48), _log_int(rng, 64, 40000)
        window, sinks = rng.choice([(0, 0), (_log_int(rng, 64, 8192), rng.choice([0, 1, 4, 64, 128]))])
        prefix = 0
    else:
        batch, prefix = _log_int(rng, 2, 96), _log_int(rng, 64, 40000)
        length, window, sinks = prefix + _log_int(rng, 1, 1500), 0, 0
    c = _case("", op, heads, group, rk, rv, q_per_kv, theta, dtype, batch, length, ragged and batch > 1, page, window, sinks, prefix)
    while True:
        w = work(c)
        if w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES:
            return c
        if c["batch"] > 4:
            c["batch"] = c["batch"] * 3 // 4
        else:
            less = c["length"] // 4
            c["length"], c["prefix"] = c["length"] - less, max(0, c["prefix"] - less)


def _lens(c):
    """Rows of every sequence, one slot of a larger batch idle; all are at least as long as what they share."""
    L, B, P = c["length"], c["batch"], c["prefix"]
    if not c["ragged"]:
        return [L] * B
    lens = [L - (977 * i) % max(1, (L - P) if P else L // 2) for i in range(B)]
    if B >= 6:
        lens[4] = 0
    return lens


def _seen(c, n):
    """Rows that a sequence of n rows attends, without shared ones."""
    if c["op"] == "prefix":
        return max(0, n - c["prefix"])
    return min(n, c["sinks"] + c["window"]) if c["window"] else n


def work(case):
    c = case
    G, s, qk, H, B = c["heads"] // c["group"], c["group"], c["q_per_kv"], c["heads"], c["batch"]
    lens = _lens(c)
    alone = sum(_seen(c, n) for n in lens)                      # rows read for one sequence each ...
    live = sum(n > 0 for n in lens)
    rows = alone + c["prefix"]                                  # ... and all rows read
    pairs = alone + c["prefix"] * live                          # (query, row)
    nbytes = rows * G * (c["rk"] + c["rv"]) * 2 + G * (c["rk"] + c["rv"]) * s * D * 2 + 2 * B * H * qk * D * 2
    flops = 2.0 * rows * G * c["rk"] * s * D + 2.0 * pairs * H * qk * (D + c["rv"]) + 2.0 * live * H * qk * c["rv"] * D
    return {"bytes": nbytes, "flops": flops}


def _dtype(c):
    return {"f16": torch.float16, "bf16": torch.bfloat16}[c["dtype"]]


def _angles(c, n, device):
    w = c["theta"] ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=device) / D)
    phi = torch.arange(n, dtype=torch.float64, device=device)[:, None] * w
    return phi.cos().float(), phi.sin().float()


def _handles(c):
    """What a program keeps beside its weights: the layer's descriptor, the angle table, scratch memory, room for the output."""
    import paper_2407_21118_amd as P
    G = c["heads"] // c["group"]
    desc = P.LayerDesc(c["heads"], D, [j * c["group"] for j in range(G + 1)], [j * c["rk"] for j in range(G + 1)],
                       [j * c["rv"] for j in range(G + 1)], P.PALU_F16 if c["dtype"] == "f16" else P.PALU_BF16,
                       rope_theta=c["theta"], q_per_kv=c["q_per_kv"])
    if c["op"] == "window":
        need = P.palu_attn_paged_workspace_bytes(desc, c["batch"], c["length"], c["window"], c["sinks"])
    else:
        need = P.palu_attn_prefix_workspace_bytes(desc, c["batch"], c["prefix"], c["length"])
    return dict(desc=desc, table=P.palu_rope_table_init(c["theta"], D, c["length"]),
                workspace=torch.empty(need, dtype=torch.uint8, device="cuda"),
                out=torch.empty(c["batch"], c["heads"] * c["q_per_kv"], D, dtype=_dtype(c), device="cuda"))


def prepare(case, seed):
    c, dev, dt = case, "cuda", _dtype(case)
    g = torch.Generator(device=dev).manual_seed(seed)
    G, s, qk, H, B, page = c["heads"] // c["group"], c["group"], c["q_per_kv"], c["heads"], c["batch"], c["page"]
    lens = _lens(c)
    per_seq = -(-c["length"] // page)
    shared = c["prefix"] // page                                # whole pages that all sequences share
    n_pages = shared + B * (per_seq - shared)
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)    # pages lie in no order
    table = torch.empty(B, per_seq, dtype=torch.int32, device=dev)
    table[:, :shared] = order[:shared]
    table[:, shared:] = order[shared:].view(B, per_seq - shared)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * scale).to(dt)

    # latents of unit size with channels that fall off like the singular values they carry; keys and values of order one
    fall = lambda r: torch.linspace(1.4, 0.6, r, device=dev)  # noqa: E731
    hk, hv = (normal(n_pages, page, G * r).view(n_pages, page, G, r).mul_(fall(r)).view(n_pages, page, G * r) for r in (c["rk"], c["rv"]))
    Bk, Bv = (normal(G, r, s * D, scale=r ** -0.5).reshape(-1) for r in (c["rk"], c["rv"]))
    seq_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    cos, sin = _angles(c, c["length"], dev)
    state = dict(case=c, lens=lens, hk=hk, hv=hv, Bk=Bk, Bv=Bv, page_table=table, seq_lens=seq_lens,
                 q=normal(B, H * qk, D, scale=1.5), q_pos=(seq_lens - 1).clamp(min=0), cos=cos, sin=sin)
    if own:
        state.update(_handles(c))
    return state


def _turn(x, cos, sin):
    a, b = x[..., : D // 2], x[..., D // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _rows(s, t, b):
    """Latents of rows t (a long tensor) of sequences b, in 32 bits."""
    c = s["case"]
    at = s["page_table"].long()[b, t // c["page"]] * c["page"] + t % c["page"]
    return s["hk"].view(-1, s["hk"].shape[-1])[at].float(), s["hv"].view(-1, s["hv"].shape[-1])[at].float()


def _keys(s, hk, t):
    """Rotated keys [.., heads, 128] of latents hk [.., R] at positions t [..]."""
    c = s["case"]
    G = c["heads"] // c["group"]
    flat = hk.reshape(-1, G, c["rk"]).transpose(0, 1).contiguous()
    k = torch.bmm(flat, s["Bk"].float().view(G, c["rk"], -1)).transpose(0, 1).reshape(*t.shape, c["heads"], D)
    return _turn(k, s["cos"][t].unsqueeze(-2), s["sin"][t].unsqueeze(-2))


def _plain(s):
    c = s["case"]
    G, qk, H, B, rv = c["heads"] // c["group"], c["q_per_kv"], c["heads"], c["batch"], c["rv"]
    dev = s["q"].device
    lens = s["seq_lens"].long()
    pos = s["q_pos"].long()
    q = _turn(s["q"].float().view(B, H, qk, D), s["cos"][pos][:, None, None], s["sin"][pos][:, None, None]) / math.sqrt(D)
    scores, values = [], []
    if c["prefix"]:
        t = torch.arange(c["prefix"], device=dev)
        hk, hv = _rows(s, t, 0)
        k = _keys(s, hk, t)                                                              # [P, H, D]
        x = torch.bmm(q.permute(1, 0, 2, 3).reshape(H, B * qk, D), k.permute(1, 2, 0).contiguous())
        x = x.view(H, B, qk, -1).transpose(0, 1)
        scores.append(x.masked_fill((t >= lens[:, None])[:, None, None], -math.inf))
        values.append(hv)
    most = max(max(_seen(c, n) for n in s["lens"]), 1)
    i = torch.arange(most, device=dev)
    first = torch.zeros_like(lens) if not c["window"] else lens.clamp(max=c["sinks"])    # rows seen at the beginning ...
    rest = torch.full_like(lens, c["prefix"]) if not c["window"] else torch.maximum(first, lens - c["window"])
    t = torch.where(i < first[:, None], i, i - first[:, None] + rest[:, None])           # ... and the newest
    seen = t < lens[:, None]
    t = t.clamp(max=c["length"] - 1)
    hk, hv = _rows(s, t, torch.arange(B, device=dev)[:, None])
    k = _keys(s, hk, t)                                                                  # [B, T, H, D]
    x = torch.bmm(q.reshape(B * H, qk, D), k.permute(0, 2, 3, 1).reshape(B * H, D, most).contiguous()).view(B, H, qk, most)
    scores.append(x.masked_fill(~seen[:, None, None], -math.inf))
    values.append(hv)
    del k, x, hk
    x = torch.cat(scores, dim=-1)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1)                                                                    # [B, H, qk]
    p = p.view(B, G, -1, p.shape[-1])                                                    # rows of one group together
    alone = p[..., -most:]
    v = values[-1].view(B, most, G, rv).transpose(1, 2).reshape(B * G, most, rv)
    o = torch.bmm(alone.reshape(B * G, -1, most), v).view(B, G, -1, rv)
    if c["prefix"]:
        v = values[0].view(-1, G, rv).transpose(0, 1).contiguous()
        both = p[..., :-most].transpose(0, 1).reshape(G, -1, c["prefix"])
        o = o + torch.bmm(both, v).view(G, B, -1, rv).transpose(0, 1)
    o = o.view(B, H, qk, rv) / torch.where(total == 0, 1.0, total)[..., None]
    up = s["Bv"].float().view(G, rv, c["group"], D).transpose(1, 2).reshape(H, rv, D)
    out = torch.bmm(o.transpose(0, 1).reshape(H, B * qk, rv), up).view(H, B, qk, D).transpose(0, 1)
    return out.reshape(B, H * qk, D).to(s["q"].dtype)


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain(s)
    import paper_2407_21118_amd as P
    if c["op"] == "window":
        return P.palu_attn_paged(s["desc"], c["batch"], c["length"], s["q"], s["q_pos"], s["hk"], s["hv"], s["page_table"],
                                 s["seq_lens"], s["Bk"], s["Bv"], s["table"], c["length"], window=c["window"], n_sink=c["sinks"],
                                 out=s["out"], workspace=s["workspace"])
    return P.palu_attn_prefix(s["desc"], c["batch"], c["prefix"], c["length"], s["q"], s["q_pos"], s["hk"], s["hv"], s["page_table"],
                              s["seq_lens"], s["Bk"], s["Bv"], s["table"], c["length"], out=s["out"], workspace=s["workspace"])


def exact(case, seed):
    """Sequence by sequence and group by group in 64 bits, rotations as products of complex numbers."""
    s, c = prepare(case, seed), case
    G, n, qk, page = c["heads"] // c["group"], c["group"], c["q_per_kv"], c["page"]
    dev = s["q"].device
    w = torch.tensor([c["theta"] ** (-2.0 * f / D) for f in range(D // 2)], dtype=torch.float64, device=dev)
    out = torch.zeros(c["batch"], c["heads"], qk, D, dtype=torch.float64, device=dev)
    Bk, Bv = s["Bk"].double().view(G, c["rk"], n, D), s["Bv"].double().view(G, c["rv"], n, D)
    table = s["page_table"].cpu().numpy()
    hk, hv = s["hk"].reshape(-1, G, c["rk"]), s["hv"].reshape(-1, G, c["rv"])
    for b, L in enumerate(s["lens"]):
        t = np.arange(L)
        if c["window"]:
            t = t[(t < c["sinks"]) | (t >= L - c["window"])]
        if not len(t):
            continue
        whose = np.where(t < c["prefix"], 0, b)
        at = torch.from_numpy(table[whose, t // page].astype(np.int64) * page + t % page).to(dev)
        when = torch.from_numpy(t).to(dev).double()[:, None] * w
        turn = torch.polar(torch.ones_like(when), when)
        angle = float(max(L - 1, 0)) * w
        q = s["q"][b].double().view(G, n, qk, D)
        q = torch.complex(q[..., : D // 2], q[..., D // 2:]) * torch.polar(torch.ones_like(angle), angle)
        for j in range(G):
            key = (hk[at, j].double() @ Bk[j].reshape(c["rk"], -1)).view(-1, n, D)
            key = torch.complex(key[..., : D // 2], key[..., D // 2:]) * turn[:, None]
            for h in range(n):
                x = (q[j, h] @ key[:, h].conj().transpose(0, 1)).real / math.sqrt(D)
                out[b, j * n + h] = torch.softmax(x, -1) @ hv[at, j].double() @ Bv[j, :, h]
    return out.reshape(c["batch"], -1, D)
