"""Rows of a quantized cache written and read back (palu_quant_latent_kv, palu_dequant_latent_kv), the projection from 4-bit weights
(palu_encode_kv_w4), and a run of all of them with the attention that reads such a cache."""

import numpy as np
import pytest
import torch

import paper_2407_21118_amd as P
from oracle import palu_oracle as O
from workloads import synth

pytestmark = pytest.mark.gpu

from gpu_util import say, torch_dtype  # noqa: E402

CODE = {4: P.PALU_I4, 3: P.PALU_I3, 2: P.PALU_I2}


def make_desc(dtype="f16", k_bits=4, v_bits=4, rk=128, rv=256, groups=3, group=2, q_per_kv=1, theta=10000.0):
    act = P.PALU_F16 if dtype == "f16" else P.PALU_BF16
    return P.LayerDesc(groups * group, 128, [j * group for j in range(groups + 1)], [j * rk for j in range(groups + 1)],
                       [j * rv for j in range(groups + 1)], act, CODE.get(k_bits, act), CODE.get(v_bits, act), rope_theta=theta,
                       q_per_kv=q_per_kv)


def caches(n_rows, R, bits, fill=0xA5):
    return (torch.full((n_rows, R * bits // 8), fill, dtype=torch.uint8, device="cuda"),
            torch.full((n_rows, R // 128), 77.0, dtype=torch.float16, device="cuda"),
            torch.full((n_rows, R // 128), -77.0, dtype=torch.float16, device="cuda"))


def latents(n, R, dtype, seed, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, R, generator=g) * torch.exp(torch.randn(n, 1, generator=g)) + offset
    if n > 2:
        x[1] = 0.0                                             # blocks of one value
        x[2] = 3.25
    return x.to(torch_dtype(dtype)).cuda()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("k_bits,v_bits", [(4, 4), (3, 2), (2, 3), (0, 4), (4, 0)])
@pytest.mark.parametrize("n", [1, 2, 37, 300])
def test_written_rows_are_the_quantizers(dtype, k_bits, v_bits, n):
    """Codes, scales and zero-points equal the oracle's; rows that no number names, and those of numbers outside the cache, stay."""
    say(f"[write] {dtype} {k_bits}/{v_bits} bits, {n} rows")
    desc = make_desc(dtype, k_bits, v_bits)
    rng = np.random.default_rng(n)
    n_rows = 2 * n + 5
    dst = rng.permutation(n_rows)[:n].astype(np.int32)
    dst[n // 3::7] = [-1, n_rows, -2 ** 31, 2 ** 31 - 1][n % 4]
    hk, hv = latents(n, desc.R_k, dtype, 1), latents(n, desc.R_v, dtype, 2, offset=5.0)
    k, v = caches(n_rows, desc.R_k, k_bits or 4), caches(n_rows, desc.R_v, v_bits or 4)
    P.palu_quant_latent_kv(desc, hk, hv, *k, *v, dst_row=torch.from_numpy(dst).cuda())
    torch.cuda.synchronize()
    keep = (dst >= 0) & (dst < n_rows)
    for h, got, bits in ((hk, k, k_bits), (hv, v, v_bits)):
        want = [x.cpu().numpy().copy() for x in caches(n_rows, h.shape[1], bits or 4)]
        if bits:
            for x, y in zip(want, O.quant_latent(h.float().cpu().numpy(), bits=bits)):
                x[dst[keep]] = y[keep]
        for x, y in zip(got, want):
            assert np.array_equal(x.cpu().numpy(), y)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [4, 3, 2])
def test_strides_alignment_and_the_other_entry_point(dtype, bits):
    """Latent rows with any stride, from any element on; the same bytes as palu_quant_latent writes."""
    desc = make_desc(dtype, bits, bits)
    plain = P.LayerDesc(desc.n_heads, 128, desc.group_head_off, desc.k_rank_off, desc.v_rank_off, desc.act_dtype) if bits == 4 else desc
    n = 19
    for first, extra in ((0, 0), (8, 8), (1, 3), (2, 130), (3, 5)):
        wide = [latents(n, R + extra, dtype, 3).flatten() for R in (desc.R_k, desc.R_v)]
        wide = [torch.cat([x.new_zeros(first), x]) for x in wide]
        hk, hv = (x[first:].view(n, -1)[:, :R] for x, R in zip(wide, (desc.R_k, desc.R_v)))
        k, v = caches(n, desc.R_k, bits), caches(n, desc.R_v, bits)
        P.palu_quant_latent_kv(desc, hk, hv, *k, *v)
        for which, (h, got) in enumerate(((hk, k), (hv, v))):
            want = [x.cpu().numpy() for x in got]
            for x, y in zip(want, O.quant_latent(h.float().cpu().numpy(), bits=bits)):
                assert np.array_equal(x, y)
            if dtype == "f16" or bits == 4:
                again = caches(n, h.shape[1], bits)
                P.palu_quant_latent(plain, which, h.contiguous(), h.shape[1], n, *again)
                assert all(torch.equal(x, y) for x, y in zip(got, again))
        # read back into rows of another stride: what lies between them stays
        out = [torch.full_like(x, 123.0) for x in wide]
        ok, ov = (x[first:].view(n, -1)[:, :R] for x, R in zip(out, (desc.R_k, desc.R_v)))
        P.palu_dequant_latent_kv(desc, *k, *v, None, ok, ov)
        for o, got, held, R in ((out[0], ok, k, desc.R_k), (out[1], ov, v, desc.R_v)):
            want = torch.from_numpy(O.dequant_latent(*(x.cpu().numpy() for x in held), bits=bits)).to(got.dtype)
            assert torch.equal(got.cpu(), want)
            assert (o[:first] == 123.0).all() and (o[first:].view(n, -1)[:, R:] == 123.0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [4, 3, 2])
def test_read_back_any_scale_and_zero_point(dtype, bits):
    """(code - zero) * scale, rounded once: the 64-bit product, rounded, except where the difference takes more than 24 bits
    (zero-points with a fraction beside large codes have 15 at most), so bit for bit."""
    desc = make_desc(dtype, bits, bits, rk=256, rv=128)
    rng = np.random.default_rng(bits)
    n_rows, n = 50, 333
    held = []
    for R in (desc.R_k, desc.R_v):
        codes = rng.integers(0, 256, (n_rows, R * bits // 8)).astype(np.uint8)
        s = (10.0 ** rng.uniform(-7, 3, (n_rows, R // 128)) * rng.choice([1, -1], (n_rows, R // 128))).astype(np.float16)
        z = rng.choice([0, 7, 7.5, -3.25, 2047, -2048, 60000, -65504, 0.125], (n_rows, R // 128)).astype(np.float16)
        s[3], z[4], s[5] = np.nan, np.nan, np.inf
        held.append((codes, s, z))
    src = rng.integers(0, n_rows, n).astype(np.int32)                  # rows may be read more than once
    src[::11] = -1
    src[5::11] = n_rows
    out = [torch.full((n, R), 55.0, dtype=torch_dtype(dtype), device="cuda") for R in (desc.R_k, desc.R_v)]
    dev = [[torch.from_numpy(x).cuda() for x in h] for h in held]
    P.palu_dequant_latent_kv(desc, *dev[0], *dev[1], torch.from_numpy(src).cuda(), *out)
    keep = (src >= 0) & (src < n_rows)
    for got, h in zip(out, held):
        with np.errstate(invalid="ignore", over="ignore"):
            want = torch.full(got.shape, 55.0, dtype=got.dtype)
            want[torch.from_numpy(keep)] = torch.from_numpy(O.dequant_latent(*h, bits=bits)[src[keep]]).to(got.dtype)
        assert torch.equal(torch.nan_to_num(got.cpu(), nan=1234.0), torch.nan_to_num(want, nan=1234.0))


def rounded_once(x, dtype):
    """64-bit numbers in the type: by way of float32 numbers whose last bit is set wherever they are inexact, which no second rounding can take
    for a tie."""
    with np.errstate(over="ignore", invalid="ignore"):
        f = x.astype(np.float32)
        u, to = f.view(np.uint32).copy(), np.abs(x) > np.abs(f.astype(np.float64))
        even = (f.astype(np.float64) != x) & np.isfinite(x) & (u & 1 == 0)
    u = np.where(even, np.where(to, u + 1, u - 1), u).astype(np.uint32)
    return torch.from_numpy(u.view(np.float32)).to(torch_dtype(dtype))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [4, 3, 2])
def test_read_back_is_rounded_once(dtype, bits):
    """Zero-points with fractions of any size, and large ones: the product takes up to 39 bits, and float32 numbers that were rounded to ties of the
    layer's type would be rounded twice."""
    desc = make_desc(dtype, bits, bits, rk=1024, rv=1024, groups=4)
    rng = np.random.default_rng(bits)
    n, R = 1500, desc.R_k
    codes = rng.integers(0, 256, (n, R * bits // 8)).astype(np.uint8)
    s = (10.0 ** rng.uniform(-3, 1, (n, R // 128)) * rng.choice([1, -1], (n, R // 128))).astype(np.float16)
    z = np.concatenate([rng.uniform(0.001, 0.2, (n // 2, R // 128)), 10.0 ** rng.uniform(-7, 4.8, (n - n // 2, R // 128)) *
                        rng.choice([1, -1], (n - n // 2, R // 128))]).astype(np.float16)
    codes[0, :64] = 0xBB                                       # 11 - 0.14978 times 0.88672: 9.6171875 in float16, 9.625 by way of float32
    s[0, 0], z[0, 0] = 0.88671875, 0.1497802734375
    s[1], z[2], s[3, :8], s[4, 3] = np.inf, np.nan, -np.inf, np.nan
    dev = [torch.from_numpy(x).cuda() for x in (codes, s, z)]
    out = [torch.empty(n, R, dtype=torch_dtype(dtype), device="cuda") for _ in range(2)]
    P.palu_dequant_latent_kv(desc, *dev, *dev, None, *out)
    with np.errstate(invalid="ignore"):
        want = torch.nan_to_num(rounded_once(O.dequant_latent(codes, s, z, bits=bits), dtype), nan=1234.0)
    for got in out:
        got = torch.nan_to_num(got.cpu(), nan=1234.0)
        say(f"[read] {dtype} {bits} bits: {int((got != want).sum())} of {want.numel()} differ")
        assert torch.equal(got, want)


def test_no_rows_at_all():
    desc = make_desc()
    k, v = caches(4, desc.R_k, 4), caches(4, desc.R_v, 4)
    none = [torch.empty(0, R, dtype=torch.float16, device="cuda") for R in (desc.R_k, desc.R_v)]
    P.palu_quant_latent_kv(desc, *none, *k, *v, dst_row=torch.empty(0, dtype=torch.int32, device="cuda"))
    P.palu_dequant_latent_kv(desc, *k, *v, None, *none)
    torch.cuda.synchronize()
    assert (k[0] == 0xA5).all() and (v[0] == 0xA5).all()


def test_many_rows_and_offsets_beyond_32_bits():
    """A cache of 4.7 GB of codes per side, written and read at its end; 40000 rows in one call."""
    desc = make_desc(rk=1024, rv=1024, groups=4, group=8)
    n_rows, n = 2300000, 40000
    k, v = ([torch.empty(n_rows, w, dtype=dt, device="cuda") for w, dt in ((2048, torch.uint8), (32, torch.float16), (32, torch.float16))]
            for _ in range(2))
    rows = torch.arange(n_rows - n, n_rows, dtype=torch.int32, device="cuda").flip(0)
    hk, hv = latents(n, 4096, "f16", 5), latents(n, 4096, "f16", 6)
    P.palu_quant_latent_kv(desc, hk, hv, *k, *v, dst_row=rows)
    ok, ov = torch.empty_like(hk), torch.empty_like(hv)
    P.palu_dequant_latent_kv(desc, *k, *v, rows, ok, ov)
    pick = torch.tensor([0, 1, 2, 777, n - 1])
    for h, o in ((hk, ok), (hv, ov)):
        held = O.quant_latent(h[pick].float().cpu().numpy())
        assert torch.equal(o[pick].cpu(), torch.from_numpy(O.dequant_latent(*held)).half())


@pytest.mark.parametrize("bits", [4, 3, 2])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_written_rows_of_every_size_of_number(dtype, bits):
    """Numbers of all exponents beside one another, blocks whose range is infinite: the oracle's float32 steps, bit for bit."""
    R, n = 256, 1500
    rng = np.random.default_rng(bits)
    raw = torch.from_numpy(rng.integers(0, 2 ** 16, (n, R)).astype(np.uint16).view(np.int16)).view(torch_dtype(dtype))
    raw = torch.where(torch.isfinite(raw), raw, torch.ones_like(raw))
    lane = np.arange(R)
    for i in range(200):                                       # blocks of a few exponents only
        keep = torch.from_numpy(rng.integers(-12, 13, R).astype(np.float32) * np.float32(2.0) ** rng.integers(-24, 15) * (1 + lane % 7))
        raw[i] = keep.to(raw.dtype).nan_to_num(0.0, 6e4, -6e4)
    desc = make_desc(dtype, bits, bits, rk=R, rv=R, groups=1)
    x = raw.cuda()
    k, v = caches(n, R, bits), caches(n, R, bits)
    P.palu_quant_latent_kv(desc, x, x, *k, *v)
    with np.errstate(over="ignore", invalid="ignore"):
        want = O.quant_latent(raw.float().numpy(), bits=bits)
    for a, b, c in zip(k, v, want):
        a, b = a.cpu().numpy(), b.cpu().numpy()
        assert np.array_equal(a.view(np.uint8), c.view(np.uint8)) and np.array_equal(a.view(np.uint8), b.view(np.uint8))


@pytest.mark.parametrize("bits", [4, 3, 2])
def test_written_rows_that_are_not_finite(bits):
    """NaN and infinities among the latents: the bytes of palu_quant_latent."""
    R, n = 256, 300
    rng = np.random.default_rng(bits)
    x = rng.standard_normal((n, R)).astype(np.float16)
    for value in (np.nan, np.inf, -np.inf):
        x[rng.random((n, R)) < 0.01] = value
    x[0], x[1, :128], x[2, :128], x[3] = np.nan, np.inf, -np.inf, rng.choice([np.nan, np.inf], R)
    desc = make_desc("f16", bits, bits, rk=R, rv=R, groups=1)
    h = torch.from_numpy(x).cuda()
    k, v, want = caches(n, R, bits), caches(n, R, bits), caches(n, R, bits)
    P.palu_quant_latent_kv(desc, h, h, *k, *v)
    P.palu_quant_latent(desc, 0, h, R, n, *want)
    for a, b, c in zip(k, v, want):
        assert torch.equal(a.view(torch.uint8), c.view(torch.uint8)) and torch.equal(b.view(torch.uint8), c.view(torch.uint8))


# ---- the projection

def weights(R, d, seed, shape="normal"):
    rng = np.random.default_rng(seed)
    codes, s, z = O.quant_latent((rng.standard_normal((R, d)) / np.sqrt(d)).astype(np.float16))
    if shape == "any":
        s = (s * 10.0 ** rng.uniform(-3, 0.3, s.shape) * rng.choice([1, -1], s.shape)).astype(np.float16)
        z = rng.choice([0, 8, 7.5, -300, 2049, 15], z.shape).astype(np.float16)
    return codes, s, z


def hold_projection(got, x, w, dtype):
    """Half a step of the result (2^-11, bfloat16 2^-8), and float32 sums: of 128 products and their zero-point's share each, then over
    the groups of 128 inputs, every addition off by at most 2^-24 of what has been added up in magnitude; in bfloat16 codes enter as
    128 + c.  Sums from 65520 on, half a step above the largest float16 number 65504, round to infinity."""
    codes = O.unpack_int4(w[0]).astype(np.float64)
    s, z = (np.repeat(np.asarray(y, np.float64), 128, axis=1) for y in w[1:])
    x = x.double().cpu().numpy()
    ref = x @ ((codes - z) * s).T
    offset = 128.0 if dtype == "bf16" else 0.0
    size = np.abs(x) @ ((codes + np.abs(z) + 2 * offset) * np.abs(s)).T
    room = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -11) * np.abs(ref) + (128 + x.shape[1] // 128 + 4) * 2.0 ** -24 * size + 2.0 ** -25
    got = got.double().cpu().numpy()
    too_large = np.isinf(got) & (np.sign(got) == np.sign(ref)) & (dtype == "f16") & (np.abs(ref) + room >= 65520.0)
    off = np.where(too_large, 0.0, np.abs(got - ref))
    say(f"    worst element at {float((off / room).max()):.3f} of its tolerance")
    assert (off <= room).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 64, 65, 130, 257])
def test_projection_of_tokens(dtype, n):
    say(f"[project] {dtype} {n} tokens")
    desc = make_desc(dtype, rk=128, rv=256, groups=2, group=4)
    d = desc.n_q_heads * 128
    x = latents(n, d, dtype, n)
    Ak, Av = weights(desc.R_k, d, 1), weights(desc.R_v, d, 2)
    out = [torch.full((n, R), float("nan"), dtype=x.dtype, device="cuda") for R in (desc.R_k, desc.R_v)]
    P.palu_encode_kv_w4(desc, x, *(torch.from_numpy(y).cuda() for y in Ak + Av), out[0], desc.R_k, out[1], desc.R_v)
    for got, w in zip(out, (Ak, Av)):
        hold_projection(got, x, w, dtype)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,q_per_kv,k_off,v_off", [(1, 1, [0, 32], [0, 96]), (3, 1, [0, 160], [0, 32]), (8, 4, [0, 512], [0, 544]), (5, 3, [0, 64], [0, 352])])
def test_projection_of_layers(dtype, heads, q_per_kv, k_off, v_off):
    """Widths of odd multiples, rows in any order with gaps between them, padding left out; any scales and zero-points."""
    say(f"[project] {dtype} {heads} x {q_per_kv} heads, ranks {k_off[1]} and {v_off[1]}")
    desc = P.LayerDesc(heads, 128, [0, heads], k_off, v_off, P.PALU_F16 if dtype == "f16" else P.PALU_BF16, q_per_kv=q_per_kv)
    d = heads * q_per_kv * 128
    for n in (1, 7, 50):
        x = latents(n, d, dtype, n)
        Ak, Av = weights(desc.R_k, d, 3, "any"), weights(desc.R_v, d, 4, "any")
        rng = np.random.default_rng(n)
        dst = rng.permutation(2 * n).astype(np.int32)[:n]
        dst[n // 2::5] = -1
        strides = (desc.R_k + 3, desc.R_v + 64)
        out = [torch.full((2 * n, w), 99.0, dtype=x.dtype, device="cuda") for w in strides]
        P.palu_encode_kv_w4(desc, x, *(torch.from_numpy(y).cuda() for y in Ak + Av), out[0], strides[0], out[1], strides[1],
                            dst_row=torch.from_numpy(dst).cuda())
        keep = dst >= 0
        for got, w, R in ((out[0], Ak, desc.R_k), (out[1], Av, desc.R_v)):
            if keep.any():
                hold_projection(got[torch.from_numpy(dst[keep]).long().cuda(), :R], x[torch.from_numpy(keep).cuda()], w, dtype)
            rest = np.ones(2 * n, bool)
            rest[dst[keep]] = False
            assert (got[torch.from_numpy(rest).cuda()] == 99.0).all() and (got[:, R:] == 99.0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,n", [(3, 513), (4, 700), (8, 609), (1, 540)])
def test_projection_of_many_tokens(dtype, heads, n):
    """Sixty-four columns a workgroup; scales and zero-points on no more than their own two bytes' alignment, one to eight groups of inputs."""
    say(f"[project] {dtype} {heads} heads, {n} tokens")
    desc = P.LayerDesc(heads, 128, [0, heads], [0, 512], [0, 576], P.PALU_F16 if dtype == "f16" else P.PALU_BF16)
    d = heads * 128
    x = latents(n, d, dtype, n)
    Ak, Av = weights(desc.R_k, d, 6, "any"), weights(desc.R_v, d, 7, "any")
    for odd in (0, 1):
        dev = []
        for y in Ak + Av:
            y = torch.from_numpy(y)
            if odd and y.dtype == torch.float16:
                y = torch.cat([y.flatten()[:1], y.flatten()]).cuda()[1:].view(y.shape)
            dev.append(y.cuda())
        dst = np.arange(n, dtype=np.int32)
        dst[::9] = -1
        out = [torch.full((n, R), 99.0, dtype=x.dtype, device="cuda") for R in (desc.R_k, desc.R_v)]
        P.palu_encode_kv_w4(desc, x, *dev, out[0], desc.R_k, out[1], desc.R_v, dst_row=torch.from_numpy(dst).cuda())
        keep = torch.from_numpy(dst >= 0).cuda()
        for got, w in zip(out, (Ak, Av)):
            hold_projection(got[keep], x[keep], w, dtype)
            assert (got[~keep] == 99.0).all()


def test_projection_beyond_the_types_middle():
    """Inputs of every size that the type has beside one another: small ones count where the large ones are zero."""
    desc = make_desc("f16", rk=128, rv=128, groups=1, group=2)
    d = 256
    x = torch.zeros(3, d, dtype=torch.float16, device="cuda")
    x[0] = torch.logspace(-7, 4, d).half()
    x[1, :40] = 6e-8                                           # the smallest numbers of the type
    x[2, 128:] = 60000.0
    w = weights(128, d, 5)
    out = [torch.empty(3, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    dev = [torch.from_numpy(y).cuda() for y in w]
    P.palu_encode_kv_w4(desc, x, *dev, *dev, out[0], 128, out[1], 128)
    hold_projection(out[0], x, w, "f16")
    assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 20, 600])
@pytest.mark.parametrize("large", [0, 1, 15])
def test_small_products_beside_large_ones_that_cancel(dtype, n, large):
    """Every token has one large input, its negative and one 2^-14.2 of it, at places that differ from token to token; the weights of the
    large two are equal.  Sums of three products are two float32 additions, off by 2^-23 of the largest magnitude each where bits are cut
    off; codes enter as 16 + c, so that magnitude is 31 inputs for the products and 16 for the zero-point's share."""
    desc = P.LayerDesc(2, 128, [0, 2], [0, 64], [0, 64], P.PALU_F16 if dtype == "f16" else P.PALU_BF16)
    d, top = 256, 4096.0
    x, codes = torch.zeros(n, d, dtype=torch.float64), np.full((64, d), large, np.uint8)
    small = torch.tensor(top * 2.0 ** -14.2).to(torch_dtype(dtype)).double()
    rng = np.random.default_rng(large)
    ones = rng.choice(d, 40, replace=False)                    # inputs whose weights are 1
    codes[:, ones] = 1
    for t in range(n):
        a, b = rng.choice([i for i in range(128) if i not in ones], 2, replace=False)
        x[t, a], x[t, b], x[t, rng.choice(ones)] = top, -top, small
    w = (codes[:, 0::2] | codes[:, 1::2] << 4, np.ones((64, 2), np.float16), np.zeros((64, 2), np.float16))
    dev = [torch.from_numpy(np.ascontiguousarray(y)).cuda() for y in w]
    out = [torch.empty(n, 64, dtype=torch_dtype(dtype), device="cuda") for _ in range(2)]
    P.palu_encode_kv_w4(desc, x.to(torch_dtype(dtype)).cuda(), *dev, *dev, out[0], 64, out[1], 64)
    room = 2 * 2.0 ** -23 * (31 + 16) * top + (2.0 ** -11 if dtype == "f16" else 2.0 ** -8) * small
    for got in out:
        off = (got.double().cpu() - small).abs().max()
        say(f"[project] {dtype} {n} tokens, weights {large}: off by {float(off):.4f} of {float(small):.4f}, tolerance {float(room):.4f}")
        assert off <= room


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [3, 40, 600])
def test_projection_of_numbers_that_are_not_finite(dtype, n):
    """A token's NaN or infinity stays in its row, a scale's or zero-point's in its channel."""
    desc = make_desc(dtype, rk=128, rv=128, groups=1, group=4)
    d = desc.n_q_heads * 128
    x = latents(n, d, dtype, 5)
    w = weights(128, d, 8)
    dev = [torch.from_numpy(y).cuda() for y in w]

    def run(x, w):
        out = [torch.empty(n, 128, dtype=x.dtype, device="cuda") for _ in "kv"]
        P.palu_encode_kv_w4(desc, x, *w, *dev, out[0], 128, out[1], 128)
        return out

    plain = run(x, dev)
    for value in (float("nan"), float("inf"), -float("inf")):
        y = x.clone()
        y[2, 77] = value
        for got, want in zip(run(y, dev), plain):
            assert not got[2].isfinite().any() and torch.equal(got[:2], want[:2]) and torch.equal(got[3:], want[3:])
        for which in (1, 2):
            other = [z.clone() for z in dev]
            other[which][17, 1] = value
            (got, same), (want, _) = run(x, other), plain
            assert not got[:, 17][x[:, 128:256].any(1)].isfinite().any() and torch.equal(same, plain[1])
            assert torch.equal(got[:, :17], want[:, :17]) and torch.equal(got[:, 18:], want[:, 18:])


# ---- as they are used together

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("q_per_kv", [1, 4])
def test_project_write_attend_read_back_in_a_graph(dtype, q_per_kv):
    """A prompt and four decode steps of three sequences, one of which pauses in the second: tokens are projected from 4-bit weights,
    quantised into pages, attended, and read back.  The steps are replays of one graph."""
    desc = make_desc(dtype, rk=256, rv=128, groups=2, group=4, q_per_kv=q_per_kv)
    B, pr, prompt, steps = 3, 16, 45, 4
    d, max_len = desc.n_q_heads * 128, prompt + steps
    g = torch.Generator(device="cuda").manual_seed(14)
    act = torch_dtype(dtype)
    rand = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(act)  # noqa: E731
    host = weights(desc.R_k, d, 1) + weights(desc.R_v, d, 2)
    w = [torch.from_numpy(y).cuda() for y in host]
    Bk, Bv = (rand(n, scale=r ** -0.5) for n, r in zip(desc.b_elems, (256, 128)))
    pages = -(-max_len // pr)
    table = torch.randperm(B * pages, generator=g, device="cuda").to(torch.int32).view(B, pages)
    pool = [tuple(x.view(B * pages, pr, -1) for x in caches(B * pages * pr, R, 4)) for R in (desc.R_k, desc.R_v)]
    rope = P.palu_rope_table_init(desc.rope_theta, 128, max_len)
    row = lambda b, t: int(table[b, t // pr]) * pr + t % pr  # noqa: E731

    x, rows = rand(B * prompt, d), torch.tensor([row(b, t) for b in range(B) for t in range(prompt)], dtype=torch.int32, device="cuda")
    h = [torch.empty(B * prompt, R, dtype=act, device="cuda") for R in (desc.R_k, desc.R_v)]
    P.palu_encode_kv_w4(desc, x, *w, h[0], desc.R_k, h[1], desc.R_v)
    for got, ww in zip(h, (host[:3], host[3:])):
        hold_projection(got, x, ww, dtype)
    P.palu_quant_latent_kv(desc, *h, *pool[0], *pool[1], dst_row=rows)

    xs, q = rand(B, d), rand(B, desc.n_q_heads, 128)
    dst = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    lens = torch.full((B,), prompt, dtype=torch.int32, device="cuda")
    new = [torch.empty(B, R, dtype=act, device="cuda") for R in (desc.R_k, desc.R_v)]
    back = [torch.zeros(B, R, dtype=act, device="cuda") for R in (desc.R_k, desc.R_v)]
    out = torch.empty(B, desc.n_q_heads, 128, dtype=act, device="cuda")
    work = torch.empty(P.palu_attn_paged_quant_workspace_bytes(desc, B, max_len), dtype=torch.uint8, device="cuda")

    def step():
        P.palu_encode_kv_w4(desc, xs, *w, new[0], desc.R_k, new[1], desc.R_v)
        P.palu_quant_latent_kv(desc, *new, *pool[0], *pool[1], dst_row=dst)
        P.palu_attn_paged_quant(desc, B, max_len, q, None, *pool[0], *pool[1], table, lens, Bk, Bv, rope, max_len, out=out, workspace=work)
        P.palu_dequant_latent_kv(desc, *pool[0], *pool[1], dst, *back)

    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    have = [prompt] * B
    for i in range(steps):
        live = [b for b in range(B) if not (i == 1 and b == 2)]
        dst.copy_(torch.tensor([row(b, have[b]) if b in live else -1 for b in range(B)], dtype=torch.int32))
        for b in live:
            have[b] += 1
        lens.copy_(torch.tensor([have[b] if b in live else 0 for b in range(B)], dtype=torch.int32))
        xs.copy_(rand(B, d))
        q.copy_(rand(B, desc.n_q_heads, 128))
        for y in back:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            if b not in live:
                assert not out[b].any() and not back[0][b].any()
                continue
            at = torch.tensor([row(b, t) for t in range(have[b])]).cuda()
            held = [O.dequant_latent(*(y.view(-1, y.shape[-1])[at].cpu().numpy() for y in p)) for p in pool]
            for y, hh in zip(back, held):
                assert torch.equal(y[b].cpu(), torch.from_numpy(hh[-1]).to(act))
            ref = O.attn_decode(q[b:b + 1].double().cpu().numpy(), np.array([have[b] - 1]), held[0][None], held[1][None],
                                Bk.double().cpu().numpy(), Bv.double().cpu().numpy(), desc.group_head_off, desc.k_rank_off, desc.v_rank_off,
                                128, desc.rope_theta, np.arange(have[b], dtype=np.int32), None, q_per_kv)[0]
            off = np.abs(out[b].double().cpu().numpy() - ref)
            rel, share = {"f16": (2.0 ** -11, 2.0 ** -14), "bf16": (2.0 ** -8, 2.0 ** -13)}[dtype]     # (as for the attention alone)
            assert (off <= rel * np.abs(ref) + share * np.abs(ref).max(-1, keepdims=True)).all()
        eager = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
