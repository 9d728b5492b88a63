"""The operators of an attention level (group norm, 8-bit products, rotary
positions, cross attention) against their definitions in 64 bits, at the
sizes, strides and masks where they can go wrong.

u = 2^-24 is half a step of fp32 relative to the value, 2^-8 that of bf16.
Each test states its bound from the operations' roundings.
"""
import math

import pytest
import torch

from paper_2008_06967_amd import _lib, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F, H = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    return g


def randn(g, *shape, dtype=F):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def within(got, ref, bound, what=""):
    """|got - ref| <= bound element by element; NaN only where ref is NaN."""
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    bad = (got - ref).abs() > bound
    bad &= ~torch.isnan(ref) & (got != ref)
    assert not bool(bad.any()), (what, int(bad.sum()), float(((got - ref).abs() / bound)[bad].max()))


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

def rotary_ref(x, pos, sections, freq, interleaved):
    x = x.double()
    P = sum(sections)
    ax = [a for a, s in enumerate(sections) for _ in range(s)]
    t = torch.stack([pos[..., ax[j]].double() * freq[j].double() for j in range(P)], -1)[..., None, :]
    c, s = torch.cos(t), torch.sin(t)
    iu = [2 * j if interleaved else j for j in range(P)]
    iv = [2 * j + 1 if interleaved else j + P for j in range(P)]
    u, v = x[..., iu], x[..., iv]
    y, size = x.clone(), torch.zeros_like(x)
    y[..., iu], y[..., iv] = u * c - v * s, u * s + v * c
    size[..., iu] = size[..., iv] = u.abs() + v.abs()
    return y, size


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("lead,H_,D,sections,inter", [
    ((1,), 1, 2, [1], False),
    ((3, 5), 3, 7, [1, 0, 2], False),          # odd head, an empty section, one copied channel
    ((7,), 8, 64, [10, 10, 10], False),
    ((129,), 2, 48, [8, 8, 8], True),
    ((2, 33), 1, 30, [4, 5, 6], True),         # pairs that fit no wide vector
    ((4, 257), 4, 128, [16, 24, 24], False),
    ((5000,), 8, 16, [2, 2, 2, 2], False),
    ((3,), 5, 1024, [512], False),
    ((1,), 300, 96, [20, 20], True),
])
def test_rotary(gpu, dtype, lead, H_, D, sections, inter):
    """The remainder of the angle is rounded once (2 pi 2^-26), sin and cos to
    about two units, the products and their sum once each: 2^-21 of |u| + |v|
    covers them; then one rounding to the output type."""
    g = gen(D + H_)
    x = randn(g, *lead, H_, D, dtype=dtype)
    pos = randn(g, *lead, len(sections)) * 100
    p = ops.RotaryParams(sections, scale=30.0, base=500.0, interleaved=inter)
    y, size = rotary_ref(x, pos, sections, p.freq, inter)
    bound = size * 2.0 ** -21 + y.abs() * HALF[dtype] * (dtype == H)
    within(ops.rotary(x, pos, p), y, bound + 1e-30)
    # strided rows, in place, and into a strided output
    wide = randn(g, *lead, H_ + 1, D, dtype=dtype)
    xs = wide[..., 1:, :]
    xs.copy_(x)
    before = wide[..., 0, :].clone()
    assert ops.rotary(xs, pos, p, out=xs) is xs
    within(xs, y, bound + 1e-30, "in place")
    assert torch.equal(wide[..., 0, :], before)
    wide2 = torch.full((*lead, H_ + 2, D), 7.0, dtype=dtype, device="cuda")
    ops.rotary(x, pos, p, out=wide2[..., 1:-1, :])
    within(wide2[..., 1:-1, :], y, bound + 1e-30, "strided output")
    assert bool((wide2[..., 0, :] == 7).all() and (wide2[..., -1, :] == 7).all())


def test_rotary_far_positions(gpu):
    """Angles of 1e7 radians: their reduction is in 64 bits, so the bound is
    the one of near positions."""
    g = gen(3)
    x = randn(g, 500, 2, 32)
    pos = torch.randint(0, 1 << 24, (500, 2), generator=g, device="cuda").float()
    p = ops.RotaryParams([8, 8])
    y, size = rotary_ref(x, pos, [8, 8], p.freq, False)
    within(ops.rotary(x, pos, p), y, size * 2.0 ** -21)


def test_rotary_shift(gpu):
    """Products of rotated rows depend on coordinate differences only."""
    g = gen(4)
    q, k = randn(g, 64, 1, 24), randn(g, 64, 1, 24)
    a, b = randn(g, 64, 3), randn(g, 64, 3)
    p = ops.RotaryParams([4, 4, 4], base=10.0)
    s0 = (ops.rotary(q, a, p) * ops.rotary(k, b, p)).double().sum(-1)
    s1 = (ops.rotary(q, a + 2.0, p) * ops.rotary(k, b + 2.0, p)).double().sum(-1)
    # a + 2 is rounded (2^-22 of up to 8) and turns by freq <= 1: 24 products of |q k| <= 25
    assert float((s0 - s1).abs().max()) <= 24 * 25 * 2.0 ** -18


# ---------------------------------------------------------------------------
# 8-bit products
# ---------------------------------------------------------------------------

def quantize_ref(x):
    """The definition: its roundings to fp32 are exact in 64 bits."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    s, r = (a / 127.0).float(), (127.0 / a).float()
    q = torch.round((x * r.double()).float())
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    q = torch.where(bad, torch.zeros_like(q), q)
    s = torch.where(bad, torch.full_like(s, math.nan), s)
    return q.to(torch.int8), s[..., 0]


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("rows,C", [(1, 1), (3, 7), (17, 16), (130, 100), (64, 129), (33, 1024), (5, 4100),
                                    (2, 20000), (4099, 67)])
def test_quantize(gpu, dtype, rows, C):
    g = gen(rows + C)
    x = randn(g, rows, C, dtype=dtype) * torch.exp(randn(g, rows, 1) * 3).to(dtype)
    q, s = ops.quantize_int8(x)
    rq, rs = quantize_ref(x)
    assert torch.equal(q, rq) and torch.equal(s, rs)
    # a column slice of wider rows, into rows of a wider buffer: the padding is zeroed, the rest is left
    wide = randn(g, rows, C + 5, dtype=dtype)
    wide[:, 3:3 + C] = x
    buf = torch.full((rows, (C + 15) // 16 * 16 + 32), 9, dtype=torch.int8, device="cuda")
    q2, _ = ops.quantize_int8(wide[:, 3:3 + C], out=buf[:, 16:16 + C])
    assert torch.equal(q2, rq)
    pad = (C + 15) // 16 * 16
    assert bool((buf[:, 16 + C:16 + pad] == 0).all())
    assert bool((buf[:, :16] == 9).all() and (buf[:, 16 + pad:] == 9).all())


def test_quantize_special_rows(gpu):
    """Zero and tiny rows, the type's largest values, ties, infinities and NaN."""
    big = torch.finfo(F).max
    rows = [[0.0] * 5, [1e-45, 0, 0, 0, -1e-45], [2.0 ** -101, 2.0 ** -100, 0, 0, 0], [big, -big, big / 2, 1, 0],
            [127, 0.5, 1.5, -2.5, -0.5], [math.inf, 1, 2, 3, 4], [1, math.nan, 2, 3, 4], [-math.inf, math.nan, 0, 0, 0],
            [1, -0.0, 1, 1, 1]]
    x = torch.tensor(rows, device="cuda")
    q, s = ops.quantize_int8(x)
    rq, rs = quantize_ref(x)
    assert torch.equal(q, rq)
    assert torch.equal(torch.isnan(s), torch.isnan(rs)) and torch.equal(s[~torch.isnan(s)], rs[~torch.isnan(rs)])
    assert q[4].tolist() == [127, 0, 2, -2, 0]
    p = ops.Int8Params(torch.ones((3, 5), dtype=torch.int8), torch.ones(3))
    y = ops.linear_int8(x, p, relu=True)
    assert bool(torch.isnan(y[5:8]).all()) and bool(torch.isfinite(y[[0, 1, 2, 4, 8]]).all())


LINEAR = [
    (1, 1, 1), (1, 16, 8), (2, 3, 5), (7, 1024, 512), (13, 100, 40), (16, 64, 64), (17, 65, 63), (31, 4096, 130),
    (64, 33, 1000), (100, 256, 256), (128, 128, 128), (129, 127, 129), (255, 320, 257), (300, 1000, 70),
    (1023, 67, 192), (2047, 515, 384), (4096, 64, 1), (5000, 48, 600),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "i8"])
@pytest.mark.parametrize("rows,ci,co", LINEAR)
def test_linear(gpu, dtype, rows, ci, co):
    """The integer sums are exact (equal 8-bit rows on both sides); their
    conversion, two products and the addition of the bias round once each."""
    g = gen(rows + ci + co)
    W = randn(g, co, ci) / math.sqrt(ci)
    b = randn(g, co) if co % 3 else None
    p = ops.Int8Params.from_float(W, b)
    wq, ws = quantize_ref(W)
    assert torch.equal(p.W, wq) and torch.equal(p.w_scale, ws)
    x = randn(g, rows, ci, dtype=H if dtype == "bf16" else F)
    q, s = quantize_ref(x)
    acc = q.double() @ wq.double().t()
    prod = acc * s.double()[:, None] * ws.double()[None]
    ref = prod + (b.double() if b is not None else 0)
    xin, xs = (ops.int8_rows(q), s) if dtype == "i8" else (x, None)
    for relu, out in ((False, F), (True, H)):
        r = torch.clamp_min(ref, 0) if relu else ref
        bound = 4 * U * (prod.abs() + r.abs()) + (r.abs() * 2.0 ** -8 if out == H else 0)
        y = ops.linear_int8(xin, p, x_scale=xs, relu=relu, out_dtype=out)
        assert y.dtype == out
        within(y, r, bound + 1e-30)
    # a strided output; its neighbors stay
    buf = torch.full((rows, co + 3), 5.0, device="cuda")
    ops.linear_int8(xin, p, x_scale=xs, out=buf[:, 2:2 + co])
    within(buf[:, 2:2 + co], ref, 4 * U * (prod.abs() + ref.abs()) + 1e-30)
    assert bool((buf[:, :2] == 5).all() and (buf[:, 2 + co:] == 5).all())


def test_linear_extremes(gpu):
    """Every product at its largest, -128 among them, over the widest input:
    the sum passes 2^30 and stays exact in 32 bits."""
    C = 65536
    x = torch.full((5, C), -128, dtype=torch.int8, device="cuda")
    w = torch.full((3, C), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    p = ops.Int8Params(w, torch.ones(3, device="cuda"))
    y = ops.linear_int8(x, p, x_scale=torch.ones(5, device="cuda"))
    assert y[0].tolist() == [float(128 * 128 * C), float(-128 * 127 * C), float(128 * 128 * C)]
    assert bool((y == y[0]).all())


def test_linear_leading_dims_and_slices(gpu):
    """[B, N, C] inputs that are column slices of one wider buffer."""
    g = gen(9)
    wide = randn(g, 3, 50, 96)
    p = ops.Int8Params.from_float(randn(g, 24, 40))
    y = ops.linear_int8(wide[..., 20:60], p)
    assert tuple(y.shape) == (3, 50, 24)
    assert torch.equal(y, ops.linear_int8(wide[..., 20:60].contiguous(), p))
    q, s = ops.quantize_int8(wide[..., 20:60])
    assert torch.equal(y, ops.linear_int8(q, p, x_scale=s))


# ---------------------------------------------------------------------------
# group norm
# ---------------------------------------------------------------------------

def act_ref(y, act):
    if act == "relu":
        return torch.relu(y)
    if act == "silu":
        return y * torch.sigmoid(y)
    if act == "gelu":
        return 0.5 * y * torch.erfc(-y / math.sqrt(2.0))
    return y


def group_norm_ref(x, G, gamma, beta, eps, act, lens):
    """(value, normalised value before gamma and beta)"""
    B, N, C = x.shape
    y, hat = torch.zeros((2, B, N, C), dtype=torch.float64, device=x.device)
    for b in range(B):
        n = N if lens is None else min(max(int(lens[b]), 0), N)
        if n == 0:
            continue
        h = x[b, :n].double().reshape(n, G, C // G)
        var, mu = torch.var_mean(h, dim=(0, 2), keepdim=True, unbiased=False)
        h = ((h - mu) / torch.sqrt(var + eps)).reshape(n, C)
        hat[b, :n] = h
        h = h * gamma.double() if gamma is not None else h
        h = h + beta.double() if beta is not None else h
        y[b, :n] = act_ref(h, act)
    return y, hat


def group_norm_bound(y, hat, gamma, beta, out):
    """Mean and deviation come from sums of chains of at most 128 terms and
    joins of partial results: within 160 u of the spread; gamma, beta and the
    activation (its slope is at most 1.13; exp, erf and the division a few
    units) add less than 16 u of the terms."""
    ga = gamma.double().abs() if gamma is not None else 1.0
    be = beta.double().abs() if beta is not None else 0.0
    return 200 * U * ((hat.abs() + 1.0) * ga + be) + y.abs() * (HALF[out] if out == H else 0)


GN = [
    (1, 1, 1, 1), (1, 1, 8, 2), (2, 3, 6, 6), (1, 128, 128, 8), (3, 100, 48, 16), (2, 1023, 192, 32), (2, 517, 20, 4),
    (4, 64, 1024, 32), (1, 4099, 24, 3), (2, 2048, 256, 32), (1, 33, 4096, 1), (1, 20000, 16, 1), (70, 5, 12, 4),
    (2, 300, 999, 9), (1, 70000, 40, 8),
]


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("B,N,C,G", GN)
def test_group_norm(gpu, dtype, B, N, C, G):
    g = gen(B + N + C + G)
    x = (randn(g, B, N, C) * torch.exp(randn(g, C) * 0.3) + randn(g, C)).to(dtype)
    gamma, beta = 1 + 0.1 * randn(g, C), 0.1 * randn(g, C)
    lens = torch.tensor([N - (b * 7) % (N + 2) for b in range(B)], dtype=torch.int32, device="cuda")   # one may be < 0
    for act, ga, be, ln in (("none", gamma, beta, None), ("relu", None, None, lens), ("silu", gamma, None, lens),
                            ("gelu", None, beta, None)):
        y, hat = group_norm_ref(x, G, ga, be, 1e-5, act, ln)
        got = ops.group_norm(x, G, ga, be, eps=1e-5, act=act, lens=ln)
        assert got.dtype == dtype
        within(got, y, group_norm_bound(y, hat, ga, be, dtype), act)
    # strided rows in and out, the other output type
    other = H if dtype == F else F
    wide = randn(g, B, N, C + 3).to(dtype)
    wide[..., 1:1 + C] = x
    buf = torch.full((B, N, C + 2), 5.0, dtype=other, device="cuda")
    y, hat = group_norm_ref(x, G, gamma, beta, 1e-3, "none", lens)
    ops.group_norm(wide[..., 1:1 + C], G, gamma, beta, eps=1e-3, lens=lens, out=buf[..., 1:1 + C])
    within(buf[..., 1:1 + C], y, group_norm_bound(y, hat, gamma, beta, other))
    assert bool((buf[..., 0] == 5).all() and (buf[..., -1] == 5).all())


@pytest.mark.parametrize("N,C,G", [(40, 16, 4), (3000, 64, 8)])
def test_group_norm_padding_is_not_read(gpu, N, C, G):
    """Rows behind a cloud's length may hold anything; a NaN among the valid
    rows reaches its own cloud and group only; lengths outside [0, N]."""
    g = gen(N)
    x = randn(g, 5, N, C)
    lens = torch.tensor([N - 3, 0, N + 9, -4, N], dtype=torch.int32, device="cuda")
    y, hat = group_norm_ref(x, G, None, None, 1e-5, "silu", lens)
    x[0, N - 3:] = math.nan
    x[1], x[3] = math.inf, math.nan
    x[4, 7, C // G + 1] = math.nan
    y[4, :, C // G:2 * (C // G)] = math.nan
    got = ops.group_norm(x, G, act="silu", lens=lens)
    within(got, y, group_norm_bound(y, hat, None, None, F))


@pytest.mark.parametrize("N", [50, 5000])
def test_group_norm_offsets(gpu, N):
    """A mean 4000 times the spread, a group led by an outlier, a constant
    group: differences to a value of the group keep the spread's precision."""
    g = gen(5)
    x = randn(g, 1, N, 32)
    x[..., 0:8] += 4000.0
    x[0, 0, 8] = 1000.0
    x[..., 16:24] = 3.14159
    y, hat = group_norm_ref(x, 4, None, None, 1e-5, "none", None)
    # the outlier stands sqrt(n) deviations off, and so does the reference point it is
    bound = group_norm_bound(y, hat, None, None, F)
    bound[..., 8:16] *= math.sqrt(8 * N)
    within(ops.group_norm(x, 4), y, bound)


# ---------------------------------------------------------------------------
# cross attention
# ---------------------------------------------------------------------------

def attention_ref(q, k, v, k_len=None, k_mask=None, scale=None):
    """(output, sum of p |v|, largest sum of |q k| scale)"""
    B, Nq, Hq, D = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    scale = 1 / math.sqrt(D) if scale is None else scale
    o, size = torch.zeros((2, B, Nq, Hq, D), dtype=torch.float64, device=q.device)
    top = 0.0
    for b in range(B):
        ok = torch.ones(Nk, dtype=torch.bool, device=q.device)
        if k_len is not None:
            ok &= torch.arange(Nk, device=q.device) < int(k_len[b])
        if k_mask is not None:
            ok &= k_mask[b].bool()
        if not bool(ok.any()):
            continue
        for h in range(Hq):
            kh, vh = k[b, ok, h // (Hq // Hkv)].double(), v[b, ok, h // (Hq // Hkv)].double()
            qh = q[b, :, h].double()
            p = torch.softmax(qh @ kh.t() * scale, -1)
            o[b, :, h], size[b, :, h] = p @ vh, p @ vh.abs()
            top = max(top, float((qh.abs() @ kh.abs().t()).max()) * abs(scale))
    return o, size, top


def attention_bound(o, size, top, D, dtype):
    """A score is off by (D + 4) u of its terms' sum (and the fp32 form's
    products may leave out 2^-22 of them), a weight by that and the
    exponential's 2^-21, the sums by 128 u, all relative; twice, for the sum
    of the weights.  bf16 rounds each weight and the output by 2^-8."""
    e = 2 * ((D + 8) * U * top + 2.0 ** -21 + 128 * U)
    if dtype == H:
        return size * (e + 2.0 ** -8) + o.abs() * 2.0 ** -8 + 1e-30
    return size * e + 1e-30


ATTN = [
    # B, Nq, Nk, Hq, Hkv, D
    (1, 1, 1, 1, 1, 1), (1, 1, 1, 4, 2, 64), (2, 1, 33, 8, 2, 64), (3, 2, 1000, 4, 4, 32), (1, 5, 7, 3, 1, 5),
    (2, 31, 65, 2, 2, 16), (1, 64, 64, 1, 1, 128), (2, 65, 127, 6, 3, 40), (1, 130, 257, 4, 1, 96),
    (2, 257, 300, 2, 2, 80), (1, 300, 31, 8, 8, 24), (4, 100, 513, 4, 2, 33), (1, 1000, 1030, 2, 1, 64),
    (1, 3, 20000, 4, 2, 64), (1, 1, 70000, 2, 1, 128), (2, 700, 129, 1, 1, 127), (1, 17, 4097, 16, 1, 8),
    (1, 520, 260, 5, 5, 48),
]


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("B,Nq,Nk,Hq,Hkv,D", ATTN)
def test_attention(gpu, dtype, B, Nq, Nk, Hq, Hkv, D):
    g = gen(Nq + Nk + D)
    q, k, v = (randn(g, B, n, h, D, dtype=dtype) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    within(ops.cross_attention(q, k, v), *_ref_and_bound(q, k, v))
    # counts (one beyond Nk, one below 0) and a mask
    k_len = torch.tensor([[Nk + 5, Nk // 2, -1, (2 * Nk + 2) // 3][b % 4] for b in range(B)], dtype=torch.int32,
                         device="cuda")
    mask = torch.rand((B, Nk), generator=g, device="cuda") < 0.6
    within(ops.cross_attention(q, k, v, k_len=k_len), *_ref_and_bound(q, k, v, k_len=k_len), "counts")
    within(ops.cross_attention(q, k, v, k_mask=mask), *_ref_and_bound(q, k, v, k_mask=mask), "mask")
    within(ops.cross_attention(q, k, v, k_len=k_len, k_mask=mask, scale=0.3),
           *_ref_and_bound(q, k, v, k_len=k_len, k_mask=mask, scale=0.3), "both")


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("B,Nq,Nk,Hq,Hkv,D", [
    (64, 300, 70, 8, 8, 64), (64, 270, 131, 8, 8, 24), (32, 300, 65, 16, 8, 30), (64, 257, 5, 8, 8, 61),
    (16, 200, 150, 8, 4, 128), (16, 200, 64, 8, 4, 88), (16, 190, 100, 8, 4, 119), (24, 130, 193, 8, 4, 64),
    (16, 260, 70, 4, 4, 69),
])
def test_attention_many_workgroups(gpu, dtype, B, Nq, Nk, Hq, Hkv, D):
    """Enough rows for the forms that give every wave rows of its own."""
    g = gen(Nq + Nk + D)
    q, k, v = (randn(g, B, n, h, D, dtype=dtype) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    within(ops.cross_attention(q, k, v), *_ref_and_bound(q, k, v))
    k_len = torch.tensor([(Nk * (b % 9)) // 8 for b in range(B)], dtype=torch.int32, device="cuda")
    mask = torch.rand((B, Nk), generator=g, device="cuda") < 0.7
    kw = dict(k_len=k_len, k_mask=mask, scale=-0.2)
    ref, bound = _ref_and_bound(q, k, v, **kw)
    ok = mask & (torch.arange(Nk, device="cuda")[None] < k_len[:, None])
    k, v = (torch.where(ok[:, :, None, None], t, torch.full((), math.nan, dtype=dtype, device="cuda")) for t in (k, v))
    within(ops.cross_attention(q, k, v, **kw), ref, bound, "counts and mask")


@pytest.mark.parametrize("dtype", [F, H])
def test_attention_scale_zero(gpu, dtype):
    """A scale of 0 gives the mean of the valid sources."""
    g = gen(21)
    q, k, v = (randn(g, 2, n, 2, 16, dtype=dtype) for n in (3, 50, 50))
    k_len = torch.tensor([50, 20], dtype=torch.int32, device="cuda")
    o, bound = _ref_and_bound(q, k, v, k_len=k_len, scale=0.0)
    within(ops.cross_attention(q, k, v, k_len=k_len, scale=0.0), o, bound)


def _ref_and_bound(q, k, v, **kw):
    o, size, top = attention_ref(q, k, v, **kw)
    return o, attention_bound(o, size, top, q.shape[-1], q.dtype)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk", [(1, 500), (200, 90)])
def test_attention_layouts(gpu, dtype, Nq, Nk):
    """Views of one projection, head-major tensors, the filled part of a
    longer buffer, shared sources (stride 0), an unaligned start, a strided
    output."""
    g = gen(Nq)
    B, Hq, Hkv, D = 3, 4, 2, 32
    q, k, v = (randn(g, B, n, h, D, dtype=dtype) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    ref, bound = _ref_and_bound(q, k, v)
    kv = torch.cat([k, v], 2)
    within(ops.cross_attention(q, kv[:, :, :Hkv], kv[:, :, Hkv:]), ref, bound, "one projection")
    hm = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v)]
    within(ops.cross_attention(*hm), ref, bound, "head-major")
    long = torch.full((B, Nk + 77, 2 * Hkv, D), math.nan, dtype=dtype, device="cuda")
    long[:, :Nk] = kv
    within(ops.cross_attention(q, long[:, :Nk, :Hkv], long[:, :Nk, Hkv:]), ref, bound, "longer buffer")
    lens = torch.full((B,), Nk, dtype=torch.int32, device="cuda")
    within(ops.cross_attention(q, long[:, :, :Hkv], long[:, :, Hkv:], k_len=lens), ref, bound, "count in it")
    flat = torch.zeros(q.numel() + 1, dtype=dtype, device="cuda")
    odd = flat[1:].view(q.shape)
    odd.copy_(q)
    out = torch.full((B, Nq + 1, Hq + 1, D + 3), 7.0, dtype=dtype, device="cuda")
    ops.cross_attention(odd, k, v, out=out[:, 1:, 1:, 1:1 + D])
    within(out[:, 1:, 1:, 1:1 + D], ref, bound, "unaligned and strided")
    assert bool((out[:, 0] == 7).all() and (out[:, :, 0] == 7).all() and (out[..., 0] == 7).all())
    assert bool((out[..., 1 + D:] == 7).all())
    one = (k[:1].expand(B, -1, -1, -1), v[:1].expand(B, -1, -1, -1))
    within(ops.cross_attention(q, *one), *_ref_and_bound(q, *one), "shared sources")


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk", [(1, 3000), (150, 200)])
def test_attention_masked_values_never_count(gpu, dtype, Nq, Nk):
    """Infinities and NaN in k and v of sources that are not valid; clouds
    without any valid source; no sources at all."""
    g = gen(7)
    B, Hq, Hkv, D = 4, 4, 2, 64
    q, k, v = (randn(g, B, n, h, D, dtype=dtype) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    mask = torch.rand((B, Nk), generator=g, device="cuda") < 0.5
    mask[1] = False
    k_len = torch.tensor([Nk - 11, Nk, Nk - 64, 0], dtype=torch.int32, device="cuda")
    ref, bound = _ref_and_bound(q, k, v, k_len=k_len, k_mask=mask)
    ok = mask & (torch.arange(Nk, device="cuda")[None] < k_len[:, None])
    bad = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(dtype).min], device="cuda").to(dtype)
    fill = bad[torch.randint(0, 4, (B, Nk, 1, 1), generator=g, device="cuda")]
    k = torch.where(ok[:, :, None, None], k, fill)
    v = torch.where(ok[:, :, None, None], v, fill)
    got = ops.cross_attention(q, k, v, k_len=k_len, k_mask=mask)
    within(got, ref, bound)
    assert bool((got[1] == 0).all() and (got[3] == 0).all())
    z = ops.cross_attention(q, k[:, :0], v[:, :0])
    assert tuple(z.shape) == tuple(q.shape) and bool((z == 0).all())
    assert ops.cross_attention(q[:, :0], k, v).numel() == 0 and ops.cross_attention(q[:0], k[:0], v[:0]).numel() == 0


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk", [(2, 2500), (140, 300)])
def test_attention_extreme_scores(gpu, dtype, Nq, Nk):
    """Scores of thousands, the largest late or early (the running maximum
    moves by more than exp can hold)."""
    g = gen(8)
    q, k, v = randn(g, 2, Nq, 2, 32, dtype=dtype), randn(g, 2, Nk, 2, 32, dtype=dtype), randn(g, 2, Nk, 2, 32, dtype=dtype)
    ramp = torch.linspace(-1, 1, Nk, device="cuda")[None, :, None, None]
    for r in (ramp, -ramp):
        k2 = (k.float() + 300.0 * r).to(dtype)
        q2 = (q.float().abs() + 1).to(dtype)
        o, size, top = attention_ref(q2, k2, v)
        within(ops.cross_attention(q2, k2, v), o, attention_bound(o, size, top, 32, dtype))


@pytest.mark.parametrize("dtype", [F, H])
def test_attention_nan_query(gpu, dtype):
    """A NaN in a query's row reaches that query and head only."""
    g = gen(10)
    q, k, v = (randn(g, 1, n, h, 32, dtype=dtype) for n, h in ((70, 2), (90, 1), (90, 1)))
    ref = ops.cross_attention(q, k, v)
    q[0, 33, 1, 5] = math.nan
    got = ops.cross_attention(q, k, v)
    assert bool(torch.isnan(got[0, 33, 1]).all())
    got[0, 33, 1] = ref[0, 33, 1]
    assert torch.equal(got, ref)


def test_empty_inputs(gpu):
    """No rows, no points, no clouds: empty results of the right shapes."""
    p = ops.Int8Params.from_float(torch.ones((4, 5), device="cuda"))
    r = ops.RotaryParams([2])
    for lead in ((0,), (0, 3), (2, 0)):
        x = torch.zeros(lead + (5,), device="cuda")
        assert tuple(ops.linear_int8(x, p).shape) == lead + (4,)
        q, s = ops.quantize_int8(x)
        assert tuple(q.shape) == lead + (5,) and tuple(s.shape) == lead
        assert tuple(ops.linear_int8(q, p, x_scale=s).shape) == lead + (4,)
        z = torch.zeros(lead + (3, 6), device="cuda")
        assert ops.rotary(z, torch.zeros(lead + (1,), device="cuda"), r).shape == z.shape
    for shape in ((0, 5, 8), (3, 0, 8)):
        assert tuple(ops.group_norm(torch.zeros(shape, device="cuda"), 2).shape) == shape


# ---------------------------------------------------------------------------
# together, streams, graphs
# ---------------------------------------------------------------------------

class Level:
    """An attention level as a program would build it: the coarse points'
    features move to the fine points."""

    def __init__(self, g, C=96, heads=4, kv=2, D=32):
        self.heads, self.kv, self.D = heads, kv, D
        mk = lambda co, ci: ops.Int8Params.from_float(randn(g, co, ci) / math.sqrt(ci), 0.1 * randn(g, co))
        self.wq, self.wkv, self.wo = mk(heads * D, C), mk(2 * kv * D, C), mk(C, heads * D)
        self.gamma, self.beta = 1 + 0.1 * randn(g, C), 0.1 * randn(g, C)
        self.rot = ops.RotaryParams([5, 5, 5], base=100.0, scale=3.0)

    def stages(self, fine, xyz_f, coarse, xyz_c, lens):
        B, N, _ = fine.shape
        M, D = coarse.shape[1], self.D
        s = {}
        s["nf"] = ops.group_norm(fine, 8, self.gamma, self.beta, act="silu")
        s["nc"] = ops.group_norm(coarse, 8, self.gamma, self.beta, act="silu", lens=lens)
        s["q"] = ops.linear_int8(s["nf"], self.wq, out_dtype=H).view(B, N, self.heads, D)
        s["kv"] = ops.linear_int8(s["nc"], self.wkv, out_dtype=H).view(B, M, 2 * self.kv, D)
        s["rq"] = ops.rotary(s["q"], xyz_f, self.rot)
        s["rk"] = ops.rotary(s["kv"][:, :, :self.kv], xyz_c, self.rot)
        s["o"] = ops.cross_attention(s["rq"], s["rk"], s["kv"][:, :, self.kv:], k_len=lens)
        s["y"] = ops.linear_int8(s["o"].reshape(B, N, -1), self.wo)
        return s


def level_inputs(g, B=3, N=333, M=90, C=96):
    return [randn(g, B, N, C), randn(g, B, N, 3), randn(g, B, M, C), randn(g, B, M, 3),
            torch.tensor([M, M // 2, 1][:B], dtype=torch.int32, device="cuda")]


def test_level_stage_by_stage(gpu):
    """The operators run together; every stage against its definition on the
    values that the stage before gave."""
    g = gen(11)
    lv = Level(g)
    fine, xf, coarse, xc, lens = a = level_inputs(g)
    s = lv.stages(*a)
    for x, key, ln in ((fine, "nf", None), (coarse, "nc", lens)):
        y, hat = group_norm_ref(x, 8, lv.gamma, lv.beta, 1e-5, "silu", ln)
        within(s[key], y, group_norm_bound(y, hat, lv.gamma, lv.beta, F), key)
    for x, p, key in ((s["nf"], lv.wq, "q"), (s["nc"], lv.wkv, "kv"), (s["o"].flatten(2), lv.wo, "y")):
        q, sc = quantize_ref(x)
        prod = (q.double() @ p.W.double().t()) * sc.double()[..., None] * p.w_scale.double()
        r = (prod + p.bias.double()).view(s[key].shape)
        half = 2.0 ** -8 if s[key].dtype == H else 0.0
        within(s[key], r, 4 * U * (prod.abs().view(r.shape) + r.abs()) + half * r.abs() + 1e-30, key)
    for x, pos, key in ((s["q"], xf, "rq"), (s["kv"][:, :, :lv.kv], xc, "rk")):
        y, size = rotary_ref(x, pos, lv.rot.sections, lv.rot.freq, False)
        within(s[key], y, size * 2.0 ** -21 + y.abs() * 2.0 ** -8 + 1e-30, key)
    within(s["o"], *_ref_and_bound(s["rq"], s["rk"], s["kv"][:, :, lv.kv:], k_len=lens), "o")


def test_level_in_a_graph(gpu):
    """Captured once and replayed on new values, with eager work of the same
    operators between the replays: the same results bit for bit."""
    g = gen(12)
    lv = Level(g)
    a = level_inputs(g)
    one = [t[:, :1].contiguous() if t.dim() == 3 and t is not a[2] and t is not a[3] else t for t in a]   # one query
    lv.stages(*a), lv.stages(*one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s, s1 = lv.stages(*a), lv.stages(*one)
    for i in range(4):
        new = level_inputs(gen(100 + i))
        for t, n in zip(a[:4], new[:4]):
            t.copy_(n)
        for t, n in zip(one[:2], new[:2]):
            t.copy_(n[:, :1])
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in ((s, lv.stages(*a)), (s1, lv.stages(*one))):
            for key in ref:
                assert torch.equal(got[key], ref[key]), (i, key)
        assert bool((s["y"] != 0).any())


def test_level_on_two_streams(gpu):
    """Two calls at once, each on a stream and with workspaces of its own."""
    g = gen(13)
    lv = Level(g)
    ins = [level_inputs(gen(20 + i), N=2000, M=700) for i in range(2)]
    refs = [lv.stages(*a) for a in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for a, st in zip(ins, streams):
        with torch.cuda.stream(st):
            outs.append(lv.stages(*a))
    torch.cuda.synchronize()
    for got, ref in zip(outs, refs):
        for key in ref:
            assert torch.equal(got[key], ref[key]), key


def test_runs_repeat_bit_for_bit(gpu):
    g = gen(14)
    lv = Level(g)
    a = level_inputs(g, N=1500, M=600)
    s = lv.stages(*a)
    for _ in range(3):
        t = lv.stages(*a)
        for key in s:
            assert torch.equal(s[key], t[key]), key


def test_workspaces_are_taken_as_they_come(gpu):
    """A caller's workspace, larger than needed and full of NaN bits, gives
    the same results; one that is too small is replaced."""
    g = gen(15)
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")
    small = torch.empty(1, dtype=torch.uint8, device="cuda")
    q, k, v = randn(g, 2, 2, 8, 64, dtype=H), randn(g, 2, 5000, 2, 64, dtype=H), randn(g, 2, 5000, 2, 64, dtype=H)
    x = randn(g, 2, 5000, 64)
    p = ops.Int8Params.from_float(randn(g, 48, 64))
    for f in (lambda w: ops.cross_attention(q, k, v, ws=w), lambda w: ops.linear_int8(x, p, ws=w),
              lambda w: ops.group_norm(x, 8, ws=w), lambda w: ops.linear_int8(x[0, :3], p, ws=w)):
        ref = f(None)
        assert torch.equal(f(ws), ref)
        ws.fill_(255)
        assert torch.equal(f(small), ref)


# ---------------------------------------------------------------------------
# large offsets
# ---------------------------------------------------------------------------

def test_offsets_past_32_bits(gpu):
    """Element offsets beyond 2^31 in every operator: the rows at the end of a
    buffer of more than 4 GiB."""
    n = (1 << 31) + 4096 * 64
    buf = torch.zeros(n, dtype=H, device="cuda")
    rows = buf.view(-1, 64)
    R = rows.shape[0]
    g = gen(16)
    tail = randn(g, 300, 64, dtype=H)
    rows[-300:] = tail
    # one cloud whose valid rows end the buffer
    y = ops.group_norm(rows[None], 8, eps=1e-5)
    cnt = R * 8
    h = tail.double().view(300, 8, 8)
    mu = h.sum((0, 2)) / cnt
    var = (h * h).sum((0, 2)) / cnt - mu * mu
    ref = ((h - mu[None, :, None]) / torch.sqrt(var + 1e-5)[None, :, None]).reshape(300, 64)
    within(y[0, -300:], ref, ref.abs() * 2.0 ** -7 + 1e-3)
    del y
    pos = torch.zeros((R, 1), device="cuda")
    pos[-300:] = randn(g, 300, 1)
    p = ops.RotaryParams([32])
    ref, size = rotary_ref(tail.view(300, 1, 64), pos[-300:], [32], p.freq, False)
    ops.rotary(rows.view(R, 1, 64), pos, p, out=rows.view(R, 1, 64))
    within(rows[-300:].view(300, 1, 64), ref, size * 2.0 ** -21 + ref.abs() * 2.0 ** -8 + 1e-30)
    rows[-300:] = tail
    del pos
    lw = ops.Int8Params.from_float(randn(g, 8, 64))
    y = ops.linear_int8(rows, lw, out_dtype=H)
    assert torch.equal(y[-300:], ops.linear_int8(tail, lw, out_dtype=H))
    del y
    # sources at the end of a long set: the rest is masked
    q = randn(g, 1, 3, 1, 64, dtype=H)
    mask = torch.zeros((1, R), dtype=torch.bool, device="cuda")
    mask[0, -300:] = True
    kv = rows.view(1, R, 1, 64)
    ref, bound = _ref_and_bound(q, tail.view(1, 300, 1, 64), tail.view(1, 300, 1, 64))
    within(ops.cross_attention(q, kv, kv, k_mask=mask), ref, bound)
    # queries at the end of a long set
    qs = rows.view(1, R, 1, 64)
    out = ops.cross_attention(qs, tail[:20].view(1, 20, 1, 64), tail[:20].view(1, 20, 1, 64))
    ref, bound = _ref_and_bound(tail.view(1, 300, 1, 64), tail[:20].view(1, 20, 1, 64), tail[:20].view(1, 20, 1, 64))
    within(out[:, -300:], ref, bound)


# ---------------------------------------------------------------------------
# the weights' precision
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("B,Nq,Nk,Hq,Hkv,D", [(2, 1, 50, 8, 2, 64), (1, 7, 2048, 4, 2, 128), (1, 300, 77, 2, 1, 32),
                                              (1, 40, 1000, 2, 2, 90), (32, 1, 60, 8, 8, 64), (200, 7, 40, 4, 2, 128),
                                              (64, 32, 130, 4, 4, 24)])
def test_attention_few_rows_keep_their_weights(gpu, B, Nq, Nk, Hq, Hkv, D):
    """bf16 rows that share a workgroup: the first of a weight's two bf16 parts is
    rounded down and leaves 2^-7 of it at most, the second half a step of that,
    2^-15; twice, for the sum of the weights; the output is rounded once."""
    g = gen(Nq + Nk)
    q, k, v = (randn(g, B, n, h, D, dtype=H) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    o, size, top = attention_ref(q, k, v)
    e = 2 * ((D + 8) * U * top + 2.0 ** -21 + 128 * U) + 2 * 2.0 ** -15
    within(ops.cross_attention(q, k, v), o, size * e + o.abs() * 2.0 ** -8 + 1e-30)


# ---------------------------------------------------------------------------
# values that the fp32 products' parts do not hold
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk,D", [(2, 300, 64), (140, 300, 64), (300, 90, 32), (150, 700, 128), (130, 70, 90),
                                     (1, 3000, 40), (129, 33, 31)])
@pytest.mark.parametrize("what", ["k -inf", "k lowest", "score past fp32", "v large", "v tiny", "q large", "q rows"])
def test_attention_any_values(gpu, dtype, Nq, Nk, D, what):
    """Infinite, huge and tiny values in valid sources and queries, at any
    number of rows: a source whose score is -infinity, or passes fp32's range
    downwards, weighs 0, so the reference is the one without it."""
    g = gen(Nq + Nk + D)
    B, Hq, Hkv = 2, 2, 1
    q, k, v = (randn(g, B, n, h, D, dtype=dtype) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    gone = torch.rand((B, Nk), generator=g, device="cuda") < 0.1
    gone[0, 40:] = False                            # the first cloud has them in its first tiles only
    gone[:, 0], gone[:, 1] = True, False
    c = D // 2
    extra = 0.0
    if what in ("k -inf", "k lowest"):
        q[..., c] = q[..., c].abs() + 0.5
        clean = k.clone()
        k[..., c][gone] = -math.inf if what == "k -inf" else torch.finfo(dtype).min
    elif what == "score past fp32":
        q[..., c], k[..., c] = 0.0, 0.0
        clean = (q.clone(), k.clone())
        q[..., c] = 1.003e25
        k[..., c][gone] = -1.003e25
    elif what == "q large":                         # scores of the usual size from factors far from it
        k = (k.float() * 2.0 ** -90).to(dtype)
        q = (q.float() * 2.0 ** 90).to(dtype)
        clean, gone = k, torch.zeros_like(gone)
    elif what == "q rows":                          # one query's scores are -infinity for all but one source
        clean, gone = k, torch.zeros_like(gone)
        k[..., c] = k[..., c].abs() + 0.5
        k[:, 1, :, c] = 0.0
    else:
        f = 1e28 if what == "v large" else 1e-38
        v = (v.float() * f).to(dtype)
        clean, gone = k, torch.zeros_like(gone)
        # fp32's denormal step, 2^-149: a product and a sum for each source, and bf16's for the output
        extra = 0.0 if f > 1 else (Nk * 2.0 ** -148 + (2.0 ** -133 if dtype == H else 0.0))
    if what == "score past fp32":
        ref, bound = _ref_and_bound(clean[0], clean[1], v, k_mask=~gone)
    else:
        ref, bound = _ref_and_bound(q, clean, v, k_mask=~gone)
    if what == "q rows":
        q[:, 0, :, c] = -math.inf                   # 0 x -inf is NaN: so that source is dropped instead
        mask = torch.ones((B, Nk), dtype=torch.bool, device="cuda")
        mask[:, 1] = False
        ref, bound = _ref_and_bound(torch.where(torch.isinf(q), torch.zeros_like(q), q), k, v, k_mask=mask)
        ref[:, 0], bound[:, 0] = 0.0, 0.0
        within(ops.cross_attention(q, k, v, k_mask=mask), ref, bound)
        return
    within(ops.cross_attention(q, k, v), ref, bound + extra)
@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq", [3, 200])
def test_attention_infinite_v_and_nan_sources(gpu, dtype, Nq):
    """An infinity in v reaches its own channel with its sign; a NaN in a
    valid source's v its own channel, in its k every query of the head."""
    g = gen(31)
    Nk, D = 120, 64
    q, k, v = (randn(g, 2, n, h, D, dtype=dtype) for n, h in ((Nq, 4), (Nk, 2), (Nk, 2)))
    ref, bound = _ref_and_bound(q, k, v)
    v[0, 7, 0, 3], v[1, 100, 1, 60] = math.inf, -math.inf
    v[1, 5, 0, 9] = math.nan
    k[1, 110, 1, 1] = math.nan
    ref[0, :, :2, 3], ref[1, :, :2, 9], ref[1, :, 2:] = math.inf, math.nan, math.nan
    within(ops.cross_attention(q, k, v), ref, bound)


@pytest.mark.parametrize("Nq,Nk", [(3, 200), (150, 300)])
def test_attention_tiny_v(gpu, Nq, Nk):
    """fp32 v of 1e-38 under equal weights: off by the sums' roundings and by
    fp32's denormal steps, one for each source's product and sum."""
    g = gen(32)
    q, k = torch.zeros((2, Nq, 2, 64), device="cuda"), randn(g, 2, Nk, 2, 64)
    v = randn(g, 2, Nk, 2, 64) * 1e-38
    ref, bound = _ref_and_bound(q, k, v)
    within(ops.cross_attention(q, k, v), ref, bound - 1e-30 + Nk * 2.0 ** -148)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk", [(2, 40), (2, 2000), (70, 130), (200, 90), (3000, 65)])
def test_attention_rows_without_a_weight(gpu, dtype, Nq, Nk):
    """Queries whose every score is -infinity give 0, whatever v holds."""
    g = gen(33)
    q, k, v = (randn(g, 2, n, h, 48, dtype=dtype) for n, h in ((Nq, 8), (Nk, 4), (Nk, 4)))
    q[..., 3] = q[..., 3].abs() + 0.5
    k[1, ..., 3] = -math.inf
    v[1] = torch.tensor([math.inf, -math.inf, math.nan, 1.0], device="cuda").to(dtype).repeat(12)
    ref, bound = _ref_and_bound(q[:1], k[:1], v[:1])
    got = ops.cross_attention(q, k, v)
    within(got[:1], ref, bound)
    assert bool((got[1] == 0).all())


# ---------------------------------------------------------------------------
# group norm: values far from the others
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("N,C,G", [(50, 32, 4), (1023, 192, 32), (5000, 32, 4), (16384, 64, 8), (3000, 30, 3),
                                   (400, 2064, 1), (70, 6000, 2)])
@pytest.mark.parametrize("size", [1e3, 1e4, 1e6])
def test_group_norm_outliers_and_offsets(gpu, dtype, N, C, G, size):
    """A value far from its group's others, first in the group, in the middle
    and last, a few leading rows, and an offset of all: every output is as close
    as the group's values are to their mean.  Sums of at most 200 roundings
    leave the mean off by 200 u of the values' mean distance to it, and an
    output by that, by its own distance's roundings and the deviation's."""
    g = gen(N + C)
    c = C // G
    x = randn(g, 6, N, C)
    x[0, 0, ::c] = size
    x[1, N // 2, ::c] = -size
    x[2, N - 1, c - 1::c] = size
    x[3, :5] *= size
    x[4] += size
    x[5, 0, ::c] = -size
    x[5] += 300.0
    x = x.to(dtype)
    y, hat = group_norm_ref(x, G, None, None, 1e-5, "none", None)
    mean = hat.abs().view(6, N, G, c).mean((1, 3), keepdim=True).expand(6, N, G, c).reshape(6, N, C)
    bound = 200 * U * (hat.abs() + mean) + (y.abs() * 2.0 ** -8 if dtype == H else 0)
    within(ops.group_norm(x, G), y, bound)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("B,Nq,Nk,Hq,Hkv,D", [(32, 1, 300, 8, 8, 128), (100, 1, 70, 4, 2, 64), (64, 16, 97, 4, 4, 40),
                                              (64, 8, 65, 16, 4, 96), (50, 33, 130, 4, 4, 64), (300, 1, 33, 1, 1, 7)])
def test_attention_few_rows_of_many_clouds(gpu, dtype, B, Nq, Nk, Hq, Hkv, D):
    """One query to a few of as many clouds and heads as fill the chip."""
    g = gen(B + Nq)
    q, k, v = (randn(g, B, n, h, D, dtype=dtype) for n, h in ((Nq, Hq), (Nk, Hkv), (Nk, Hkv)))
    k_len = torch.tensor([(b * 11) % (Nk + 1) for b in range(B)], dtype=torch.int32, device="cuda")
    mask = torch.rand((B, Nk), generator=g, device="cuda") < 0.7
    within(ops.cross_attention(q, k, v), *_ref_and_bound(q, k, v))
    kw = dict(k_len=k_len, k_mask=mask)
    within(ops.cross_attention(q, k, v, **kw), *_ref_and_bound(q, k, v, **kw))


# ---------------------------------------------------------------------------
# the 8-bit product's large tiles
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "i8"])
@pytest.mark.parametrize("rows,ci,co", [
    (4001, 1100, 3003),      # tiles of 256 x 256: 16 x 12 of them, 9 of 128 columns, remainders in all three
    (12289, 1040, 1025),     # 49 x 5, the last of one row and one channel
    (3000, 515, 1100),       # tiles of 128 x 128: 24 x 9, 5 of 128 columns
    (25000, 131, 67),        # 196 x 1, two of 128 columns, the second of 16
    (2500, 2000, 1409),      # 20 x 12, 16 of 128 columns
])
def test_linear_large_tiles(gpu, dtype, rows, ci, co):
    """Sizes for each of the large tiles, with several steps over the columns
    and with remainders; the bound of test_linear."""
    g = gen(rows + ci)
    W = randn(g, co, ci) / math.sqrt(ci)
    b = randn(g, co)
    p = ops.Int8Params.from_float(W, b)
    x = randn(g, rows, ci, dtype=H if dtype == "bf16" else F) * torch.exp(randn(g, rows, 1)).to(H if dtype == "bf16" else F)
    q, s = quantize_ref(x)
    wq, ws = quantize_ref(W)
    prod = (q.double() @ wq.double().t()) * s.double()[:, None] * ws.double()[None]
    xin, xs = (ops.int8_rows(q), s) if dtype == "i8" else (x, None)
    for relu, out in ((False, F), (True, H)):
        ref = prod + b.double()
        ref = torch.clamp_min(ref, 0) if relu else ref
        bound = 4 * U * (prod.abs() + ref.abs()) + (ref.abs() * 2.0 ** -8 if out == H else 0) + 1e-30
        buf = torch.full((rows + 1, co + 1), 5.0, dtype=out, device="cuda")
        ops.linear_int8(xin, p, x_scale=xs, relu=relu, out_dtype=out, out=buf[:rows, :co])
        within(buf[:rows, :co], ref, bound)
        assert bool((buf[rows] == 5).all() and (buf[:, co] == 5).all())


# ---------------------------------------------------------------------------
# outputs beside and over inputs
# ---------------------------------------------------------------------------

def test_outputs_beside_inputs(gpu):
    """Other columns or rows of an input's buffer take the output; views that
    share bytes with an input are refused."""
    g = gen(40)
    buf = randn(g, 2, 60, 96)
    x = buf[..., :32]
    for out in (buf[..., 32:64], buf[..., 64:96]):
        ref = ops.group_norm(x.clone(), 8)
        assert torch.equal(ops.group_norm(x, 8, out=out), ref)
    flat = buf.view(120, 96)
    p = ops.Int8Params.from_float(randn(g, 40, 32))
    ref = ops.linear_int8(flat[::2, :32].clone(), p)
    assert torch.equal(ops.linear_int8(flat[::2, :32], p, out=flat[::2, 32:72]), ref)
    assert torch.equal(ops.linear_int8(flat[::2, :32], p, out=flat[1::2, :40]), ref)
    r = ops.RotaryParams([8])
    pos = randn(g, 120, 1)
    h = flat.view(120, 6, 16)
    ref = ops.rotary(h[:, :2].clone(), pos, r)
    assert torch.equal(ops.rotary(h[:, :2], pos, r, out=h[:, 2:4]), ref)
    qkvo = randn(g, 2, 50, 4, 3, 16)
    q, k, v, o = (qkvo[:, :, i] for i in range(4))
    ref = ops.cross_attention(q.clone(), k, v)
    assert torch.equal(ops.cross_attention(q, k, v, out=o), ref)
    heads = randn(g, 2, 4, 50, 16).transpose(1, 2)          # clouds, points, heads: one after another
    ref = ops.cross_attention(heads[:, :, :2].clone(), k[:, :, :2], v[:, :, :2])
    assert torch.equal(ops.cross_attention(heads[:, :, :2], k[:, :, :2], v[:, :, :2], out=heads[:, :, 2:]), ref)
    before = buf.clone()
    for f in (lambda: ops.group_norm(x, 8, out=buf[..., 16:48]),
              lambda: ops.group_norm(buf[:1, :59], 8, out=buf[:1, 1:]),
              lambda: ops.linear_int8(flat[:60, :32], p, out=flat[30:90, 24:64]),
              lambda: ops.rotary(h[:119], pos[:119], r, out=h[1:]),
              lambda: ops.rotary(h[:, :2], pos, r, out=h[:, 1:3]),
              lambda: ops.cross_attention(q, k, v, out=qkvo.view(2, 50, 12, 16)[:, :, 8:11])):
        with pytest.raises(_lib.MesorasiError, match="overlaps"):
            f()
    assert torch.equal(buf, before)


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk", [(1, 700), (150, 130)])
def test_attention_shared_mask(gpu, dtype, Nq, Nk):
    """One row of a mask for all clouds, without a copy."""
    g = gen(41)
    q, k, v = (randn(g, 3, n, h, 32, dtype=dtype) for n, h in ((Nq, 4), (Nk, 2), (Nk, 2)))
    mask = (torch.rand((1, Nk), generator=g, device="cuda") < 0.5).expand(3, Nk)
    got = ops.cross_attention(q, k, v, k_mask=mask)
    within(got, *_ref_and_bound(q, k, v, k_mask=mask))
    assert torch.equal(got, ops.cross_attention(q, k, v, k_mask=mask.contiguous()))


def test_rotary_precision(gpu):
    """fp32 over many angles, in the 2-norm: the remainder's rounding (at most
    half a unit of pi / 4, uniform: 1.4e-8), sin and cos to a unit (3.4e-8), products
    (half a unit of each, 1.2e-8 of the pair) and their sum (1.7e-8) add up to
    4.3e-8 as independent errors."""
    g = gen(42)
    x, pos = randn(g, 20000, 4, 64), randn(g, 20000, 3) * 25
    p = ops.RotaryParams([10, 10, 12], base=1000.0, scale=20.0)
    y, _ = rotary_ref(x, pos, p.sections, p.freq, False)
    err = float((ops.rotary(x, pos, p).double() - y).norm() / y.norm())
    print("normwise error", err)
    assert err <= 4.8e-8


def test_rotary_quarter_turns(gpu):
    """Angles at and around every eighth of a turn, of either sign, small and
    large, and angles that are not finite."""
    g = gen(43)
    eighth = torch.arange(-64, 65, dtype=torch.float64, device="cuda") / 8
    turn = torch.cat([eighth * 2 * math.pi, (eighth + 4096) * 2 * math.pi]).float()
    pos = torch.cat([turn, torch.nextafter(turn, torch.full_like(turn, math.inf)),
                     torch.nextafter(turn, torch.full_like(turn, -math.inf)), -turn])[:, None]
    x = randn(g, pos.shape[0], 3, 6)
    p = ops.RotaryParams([3], freq=torch.tensor([1.0, -0.5, 3.0]))
    y, size = rotary_ref(x, pos, [3], p.freq, False)
    within(ops.rotary(x, pos, p), y, size * 2.0 ** -21 + 1e-30)
    pos[5], pos[6], pos[7] = math.inf, math.nan, 3e38
    z = ops.rotary(x, pos, p)
    assert bool(torch.isnan(z[5:7]).all()) and bool(torch.isfinite(z[7:]).all())


@pytest.mark.parametrize("dtype", [F, H])
@pytest.mark.parametrize("Nq,Nk", [(2, 40), (2, 2000), (70, 130), (200, 90), (3000, 65)])
def test_attention_scaled_scores_past_the_range(gpu, dtype, Nq, Nk):
    """Scores that are finite until they are scaled: -infinity weighs nothing,
    +infinity leaves no weights defined, and is no 0."""
    g = gen(44)
    q, k, v = (randn(g, 2, n, h, 48, dtype=dtype) for n, h in ((Nq, 8), (Nk, 4), (Nk, 4)))
    q, k = q.abs() + 0.5, -(k.abs() + 0.5)
    k[1, Nk // 2] *= -1.0                            # the second cloud has one source of positive scores
    got = ops.cross_attention(q, k, v, scale=1e38)
    assert bool((got[0] == 0).all()) and bool(torch.isnan(got[1]).all())
    got = ops.cross_attention(q, k, v, scale=-1e38)
    assert bool(torch.isnan(got).all())
