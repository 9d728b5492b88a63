"""The operators of an attention level as measurable cases.

An attention level moves features from one set of points to another, as the
3-NN interpolation does, with learned weights: rows are normalised, projected,
rotated by their coordinates, attended to and projected again.  The kinds:

  attention   every query point over the points of another set (another
              count), grouped heads, a count or a mask of valid points
  linear      a layer's product in 8-bit integers, one scale for each row and
              each output channel; rows come in fp32 or bf16 and are brought to
              8 bits within the call, or come as 8-bit rows already
  group_norm  group normalisation over each cloud's valid points with an
              activation, channels last
  rotary      feature pairs rotated by angles of several coordinates (x, y, z
              of points, or time, height, width)

With ``own`` unset, ``run`` computes them in elementary torch operations in 32
bits (64 for angles); with it set, through the package's public entry points.
``exact`` evaluates the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # one new point asked against two cached scenes of unequal counts: the latency of a single query
        dict(name="attention_one_query", kind="attention", B=2, Nq=1, Nk=2048, Hq=8, Hkv=2, D=64, dtype="bf16",
             ragged=True, drop=0.0),
        # an object's points over the next level's, counts that fit no tile, a tenth of the sources masked
        dict(name="attention_objects", kind="attention", B=16, Nq=1023, Nk=257, Hq=4, Hkv=4, D=32, dtype="f32",
             ragged=False, drop=0.1),
        # a room's points over a quarter of them, fp32 features of the segmentation network's kind
        dict(name="attention_rooms", kind="attention", B=4, Nq=4096, Nk=1024, Hq=8, Hkv=8, D=64, dtype="f32",
             ragged=True, drop=0.0),
        # LiDAR sweeps over their first level, grouped heads: the largest
        dict(name="attention_sweeps", kind="attention", B=4, Nq=16384, Nk=4096, Hq=8, Hkv=2, D=128, dtype="bf16",
             ragged=False, drop=0.0),
        # the classifier's first fully connected layer on a few objects
        dict(name="linear_few_rows", kind="linear", rows=13, c_in=1024, c_out=512, dtype="f32", out="f32", relu=True,
             bias=True),
        # a projection of a batch of objects' points, a row count that fits no tile
        dict(name="linear_points", kind="linear", rows=16368, c_in=320, c_out=256, dtype="f32", out="f32", relu=True,
             bias=True),
        # a wide layer on a batch of sweeps: the largest product
        dict(name="linear_wide", kind="linear", rows=16384, c_in=4096, c_out=4096, dtype="bf16", out="bf16",
             relu=False, bias=False),
        # one small object
        dict(name="group_norm_object", kind="group_norm", B=1, N=128, C=128, G=8, dtype="f32", act="relu",
             ragged=False),
        # a padded batch of objects, bf16
        dict(name="group_norm_padded", kind="group_norm", B=16, N=1023, C=192, G=32, dtype="bf16", act="silu",
             ragged=True),
        # a batch of sweeps' features: the most bytes
        dict(name="group_norm_sweeps", kind="group_norm", B=16, N=16384, C=256, G=32, dtype="f32", act="gelu",
             ragged=False),
        # a few new points' queries
        dict(name="rotary_few_points", kind="rotary", rows=7, H=8, D=64, sections="10,10,10", dtype="f32",
             interleaved=False, grid=False),
        # a batch of sweeps' queries
        dict(name="rotary_sweeps", kind="rotary", rows=65536, H=8, D=128, sections="16,24,24", dtype="bf16",
             interleaved=False, grid=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "linear", "linear", "group_norm", "rotary"])
    if kind == "attention":
        dtype = rng.choice(["f32", "bf16"])
        D = rng.choice([16, 24, 32, 40, 64, 64, 80, 96, 128])
        Hkv = rng.choice([1, 2, 3, 4, 8])
        Hq = Hkv * rng.choice([1, 1, 2, 4])
        Nk = _log(rng, 1, 16384)
        Nq = rng.choice([1, rng.randint(1, 16), _log(rng, 1, 16384)])
        # fp32 up to the work of the rooms, bf16 up to that of the sweeps
        most = 4 * 4096 * 1024 * 8 * 64 if dtype == "f32" else 4 * 16384 * 4096 * 8 * 128 // 2
        B = _log(rng, 1, 16)
        while B > 1 and (B * Nq * Nk * Hq * D > most or B * Nk * Hkv * D > 1 << 25):
            B -= 1
        while B * Nq * Nk * Hq * D > most or B * Nq * Hq * D > 1 << 25:
            Nq = (Nq + 1) // 2
        return dict(kind=kind, B=B, Nq=Nq, Nk=Nk, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, ragged=rng.random() < 0.4,
                    drop=rng.choice([0.0, 0.0, 0.1]))
    if kind == "linear":
        rows, c_in, c_out = _log(rng, 1, 65536), _log(rng, 16, 4096), _log(rng, 8, 4096)
        while rows * c_in * c_out > 16384 * 4096 * 4096 or rows * (c_in + c_out) > 1 << 26:
            rows //= 2
        return dict(kind=kind, rows=rows, c_in=c_in, c_out=c_out, dtype=rng.choice(["f32", "bf16", "i8"]),
                    out=rng.choice(["f32", "bf16"]), relu=rng.random() < 0.5, bias=rng.random() < 0.7)
    if kind == "group_norm":
        G = rng.choice([1, 4, 8, 16, 32])
        C = G * _log(rng, 1, 1024 // G)
        B, N = _log(rng, 1, 32), _log(rng, 1, 65536)
        while B * N * C > 16 * 16384 * 256:
            N = (N + 1) // 2
        return dict(kind=kind, B=B, N=N, C=C, G=G, dtype=rng.choice(["f32", "bf16"]),
                    act=rng.choice(["none", "relu", "silu", "gelu"]), ragged=rng.random() < 0.4)
    D = rng.choice([16, 24, 32, 48, 64, 96, 128])
    pairs = D // 2 - rng.choice([0, 0, 2])
    axes = rng.choice([1, 2, 3, 3, 3])
    sections = [pairs // axes] * axes
    sections[-1] += pairs - sum(sections)
    rows, H = _log(rng, 1, 65536), rng.choice([1, 2, 3, 4, 8])
    return dict(kind="rotary", rows=rows, H=H, D=D, sections=",".join(str(s) for s in sections),
                dtype=rng.choice(["f32", "bf16"]), interleaved=rng.random() < 0.3, grid=rng.random() < 0.4)


def _counts(B, N, ragged):
    """The clouds' valid counts: all N, or spread over N / 3 .. N."""
    return [N - (b * 37 * N // 100) % max(1, (2 * N) // 3) if ragged else N for b in range(B)]


def _sections(case):
    return [int(s) for s in case["sections"].split(",")]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=DEV).to(dtype)

    kind = case["kind"]
    st = dict(case)
    if kind == "attention":
        B, Nq, Nk, Hq, Hkv, D = (case[k] for k in ("B", "Nq", "Nk", "Hq", "Hkv", "D"))
        dt = TYPES[case["dtype"]]
        st["q"] = normal(B, Nq, Hq, D, dtype=dt)
        kv = normal(B, Nk, 2 * Hkv, D, dtype=dt)         # one projection's rows hold both
        st["k"], st["v"] = kv[:, :, :Hkv], kv[:, :, Hkv:]
        st["k_len"] = torch.tensor(_counts(B, Nk, True), dtype=torch.int32, device=DEV) if case["ragged"] else None
        st["k_mask"] = torch.rand((B, Nk), generator=g, device=DEV) >= case["drop"] if case["drop"] else None
        return st
    if kind == "linear":
        rows, ci, co = case["rows"], case["c_in"], case["c_out"]
        w = normal(co, ci) * math.sqrt(2.0 / ci)
        st["wq"], st["ws"] = _quantize_plain(w)
        st["b"] = torch.rand((co,), generator=g, device=DEV) * 0.2 - 0.1 if case["bias"] else None
        x = normal(rows, ci)
        # points' features differ in size from row to row
        x = x * torch.exp(normal(rows, 1) * 0.5)
        if case["dtype"] == "i8":
            st["x"], st["xs"] = _quantize_plain(x)
        else:
            st["x"], st["xs"] = x.to(TYPES[case["dtype"]]), None
        if own:
            from paper_2008_06967_amd import ops
            st["p"] = ops.Int8Params(st["wq"], st["ws"], st["b"])
            if case["dtype"] == "i8":
                st["x"] = ops.int8_rows(st["x"])
        return st
    if kind == "group_norm":
        B, N, C = case["B"], case["N"], case["C"]
        scale, shift = torch.exp(normal(C) * 0.3), normal(C) * 0.5
        st["x"] = (normal(B, N, C) * scale + shift).to(TYPES[case["dtype"]])
        st["gamma"], st["beta"] = 1.0 + 0.1 * normal(C), 0.1 * normal(C)
        st["lens"] = torch.tensor(_counts(B, N, True), dtype=torch.int32, device=DEV) if case["ragged"] else None
        return st
    rows, H, D, sec = case["rows"], case["H"], case["D"], _sections(case)
    st["x"] = normal(rows, H, D, dtype=TYPES[case["dtype"]])
    if case["grid"]:        # time, height, width counts
        st["pos"] = torch.randint(0, 1024, (rows, len(sec)), generator=g, device=DEV).float()
        st["freq"] = torch.cat([10000.0 ** (-torch.arange(s, device=DEV, dtype=torch.float64) / s) for s in sec]).float()
    else:                   # coordinates in metres, a sweep's reach
        st["pos"] = normal(rows, len(sec)) * 25.0
        st["freq"] = torch.cat([20.0 * 1000.0 ** (-torch.arange(s, device=DEV, dtype=torch.float64) / s)
                                for s in sec]).float()
    if own:
        from paper_2008_06967_amd import ops
        st["p"] = ops.RotaryParams(sec, freq=st["freq"], interleaved=case["interleaved"])
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _DISPATCH[own][state["kind"]](state)


def _own_attention(st):
    from paper_2008_06967_amd import ops
    return ops.cross_attention(st["q"], st["k"], st["v"], k_len=st["k_len"], k_mask=st["k_mask"])


def _own_linear(st):
    from paper_2008_06967_amd import ops
    return ops.linear_int8(st["x"], st["p"], x_scale=st["xs"], relu=st["relu"], out_dtype=TYPES[st["out"]])


def _own_group_norm(st):
    from paper_2008_06967_amd import ops
    return ops.group_norm(st["x"], st["G"], st["gamma"], st["beta"], eps=1e-5, act=st["act"], lens=st["lens"])


def _own_rotary(st):
    from paper_2008_06967_amd import ops
    return ops.rotary(st["x"], st["pos"], st["p"])


def _valid(st, B, Nk):
    """[B, Nk] truth values: sources a query may attend to (None: all)."""
    ok = st["k_mask"]
    if st["k_len"] is not None:
        n = torch.arange(Nk, device=DEV)[None, :] < st["k_len"][:, None]
        ok = n if ok is None else ok & n
    return ok


def _plain_attention(st):
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    B, Nq, Hq, D = q.shape
    Nk, Hkv = k.shape[1], k.shape[2]
    g = Hq // Hkv
    ok = _valid(st, B, Nk)
    # [B, Hkv, Nq * g, D]: the queries of a group of heads share their sources
    q = q.reshape(B, Nq, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Nq * g, D)
    k = k.permute(0, 2, 3, 1).contiguous()
    v = v.permute(0, 2, 1, 3).contiguous()
    if ok is not None:
        v = torch.where(ok[:, None, :, None], v, torch.zeros((), device=DEV))
    s = torch.matmul(q, k)
    s = s * (1.0 / math.sqrt(D))
    if ok is not None:
        s = torch.where(ok[:, None, None, :], s, torch.full((), -math.inf, device=DEV))
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros((), device=DEV), m)
    p = torch.exp(s - m)
    del s
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v)
    o = o / torch.where(l == 0, torch.ones((), device=DEV), l)
    return o.reshape(B, Hkv, Nq, g, D).permute(0, 2, 1, 3, 4).reshape(B, Nq, Hq, D).to(st["q"].dtype)


def _quantize_plain(x):
    x = x.float()
    a = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    top = torch.full_like(a, 127.0)
    r = top / a
    return torch.round(x * r).to(torch.int8), (a / top)[..., 0]


def _plain_linear(st):
    q, s = (st["x"], st["xs"]) if st["xs"] is not None else _quantize_plain(st["x"])
    y = torch.matmul(q.float(), st["wq"].float().t()) * s[:, None] * st["ws"][None, :]
    if st["b"] is not None:
        y = y + st["b"]
    if st["relu"]:
        y = torch.clamp_min(y, 0.0)
    return y.to(TYPES[st["out"]])


def _act(y, act):
    if act == "relu":
        return torch.clamp_min(y, 0.0)
    if act == "silu":
        return y / (1.0 + torch.exp(-y))
    if act == "gelu":
        return 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    return y


def _norm(x, st):
    """Both the 32-bit and the 64-bit value, by x's type."""
    B, N, C = x.shape
    G = st["G"]
    x = x.reshape(B, N, G, C // G)
    if st["lens"] is not None:
        ok = (torch.arange(N, device=DEV)[None, :] < st["lens"][:, None])[:, :, None, None]
        cnt = (st["lens"].to(x.dtype) * (C // G))[:, None, None, None]
        x = torch.where(ok, x, torch.zeros((), device=DEV, dtype=x.dtype))
        mu = x.sum((1, 3), keepdim=True) / cnt
        d = torch.where(ok, x - mu, torch.zeros((), device=DEV, dtype=x.dtype))
        var = (d * d).sum((1, 3), keepdim=True) / cnt
    else:
        ok = None
        d = x - x.mean((1, 3), keepdim=True)
        var = (d * d).mean((1, 3), keepdim=True)
    y = (d * torch.rsqrt(var + 1e-5)).reshape(B, N, C) * st["gamma"].to(x.dtype) + st["beta"].to(x.dtype)
    y = _act(y, st["act"])
    return y if ok is None else torch.where(ok[:, :, :, 0], y, torch.zeros((), device=DEV, dtype=y.dtype))


def _plain_group_norm(st):
    return _norm(st["x"].float(), st).to(st["x"].dtype)


def _rotate(x, st, kind):
    sec = _sections(st)
    P = sum(sec)
    axis = torch.cat([torch.full((s,), i, device=DEV, dtype=torch.int64) for i, s in enumerate(sec)])
    ang = st["pos"].double()[:, axis] * st["freq"].double()
    c, s = torch.cos(ang).to(kind)[:, None, :], torch.sin(ang).to(kind)[:, None, :]
    y = x.clone()
    if st["interleaved"]:
        u, v = x[..., 0:2 * P:2], x[..., 1:2 * P:2]
        y[..., 0:2 * P:2], y[..., 1:2 * P:2] = u * c - v * s, u * s + v * c
    else:
        u, v = x[..., :P], x[..., P:2 * P]
        y[..., :P], y[..., P:2 * P] = u * c - v * s, u * s + v * c
    return y


def _plain_rotary(st):
    return _rotate(st["x"].float(), st, torch.float32).to(st["x"].dtype)


_DISPATCH = {
    False: dict(attention=_plain_attention, linear=_plain_linear, group_norm=_plain_group_norm, rotary=_plain_rotary),
    True: dict(attention=_own_attention, linear=_own_linear, group_norm=_own_group_norm, rotary=_own_rotary),
}


def exact(case, seed):
    global own
    keep, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = keep
    kind = case["kind"]
    if kind == "group_norm":
        x = st["x"].double()
        y = torch.zeros_like(x)
        for b, n in enumerate(_counts(case["B"], case["N"], case["ragged"])):
            h = x[b, :n].reshape(n, case["G"], -1)
            var, mean = torch.var_mean(h, dim=(0, 2), keepdim=True, unbiased=False)
            h = ((h - mean) / torch.sqrt(var + 1e-5)).reshape(n, -1) * st["gamma"].double() + st["beta"].double()
            act = case["act"]
            if act == "relu":
                h = torch.where(h > 0, h, torch.zeros_like(h))
            elif act == "silu":
                h = h * torch.sigmoid(h)
            elif act == "gelu":
                h = h * 0.5 * torch.erfc(-h / math.sqrt(2.0))
            y[b, :n] = h
        return y
    if kind == "rotary":
        x, sec = st["x"].double(), _sections(case)
        y, j = x.clone(), 0
        P = sum(sec)
        for a, n in enumerate(sec):
            for i in range(n):
                t = st["pos"][:, a].double()[:, None] * st["freq"][j].double()
                u, v = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + P)
                z = torch.complex(x[..., u], x[..., v]) * torch.polar(torch.ones_like(t), t)
                y[..., u], y[..., v] = z.real, z.imag
                j += 1
        return y
    if kind == "linear":
        if st["xs"] is None:
            # the definition's roundings to 32 bits: a / 127, 127 / a and x r
            x = st["x"].double()
            a = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
            s = (a / 127.0).float().double()
            q = torch.round((x * (127.0 / a).float().double()).float().double())
        else:
            q, s = st["x"].double(), st["xs"].double()[:, None]
        y = torch.empty((case["rows"], case["c_out"]), dtype=torch.float64, device=DEV)
        w = (st["wq"].double() * st["ws"].double()[:, None]).t().contiguous()
        for r in range(0, case["rows"], 4096):
            h = (q[r:r + 4096] * s[r:r + 4096]) @ w
            if st["b"] is not None:
                h = h + st["b"].double()
            y[r:r + 4096] = torch.relu(h) if case["relu"] else h
        return y
    B, Nq, Nk, Hq, D = (case[k] for k in ("B", "Nq", "Nk", "Hq", "D"))
    g = Hq // case["Hkv"]
    o = torch.zeros((B, Nq, Hq, D), dtype=torch.float64, device=DEV)
    counts = _counts(B, Nk, case["ragged"])
    for b in range(B):
        rows = torch.arange(counts[b], device=DEV)
        if st["k_mask"] is not None:
            rows = rows[st["k_mask"][b, :counts[b]]]
        if rows.numel() == 0:
            continue
        for h in range(Hq):
            k, v = st["k"][b, rows, h // g].double(), st["v"][b, rows, h // g].double()
            for n in range(0, Nq, 8192):
                s = st["q"][b, n:n + 8192, h].double() @ k.t() / math.sqrt(D)
                o[b, n:n + 8192, h] = torch.softmax(s, -1) @ v
    return o


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "attention":
        e = 4 if case["dtype"] == "f32" else 2
        B, Nq, Hq, Hkv, D = (case[k] for k in ("B", "Nq", "Hq", "Hkv", "D"))
        n = sum(_counts(B, case["Nk"], case["ragged"])) * (1.0 - case["drop"])
        return {"bytes": int(e * D * (2 * B * Nq * Hq + 2 * n * Hkv)), "flops": int(4 * Nq * n * Hq * D)}
    if kind == "linear":
        rows, ci, co = case["rows"], case["c_in"], case["c_out"]
        return {"bytes": rows * ci * {"f32": 4, "bf16": 2, "i8": 1}[case["dtype"]] + ci * co
                + rows * co * (4 if case["out"] == "f32" else 2), "flops": 2 * rows * ci * co}
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "group_norm":
        n = sum(_counts(case["B"], case["N"], case["ragged"]))
        return {"bytes": e * case["C"] * (n + case["B"] * case["N"]), "flops": 10 * n * case["C"]}
    n = case["rows"] * case["H"] * case["D"]
    return {"bytes": 2 * e * n + 4 * case["rows"] * len(_sections(case)), "flops": 3 * n}
