"""The operators of a point network's pointwise half as measurable cases: group norm with an activation over a batch of
clouds, dropout from a counter-based generator, and linear layers in microscaled 4-bit floating point, with their gradients.

A case is a dict of plain values:
  op          norm_fwd   activation(group norm) with dropout, and the groups' statistics
              norm_bwd   their gradients
              drop_fwd   residual + dropout of a branch
              drop_bwd   the branch's gradient
              quantise   rows (or columns) to 4 bits and back
              linear     activation(x W^T + bias), x rounded to 4 bits on the way, W kept in 4 bits
              linear_bwd the gradients of x and W, what flows to the output rounded at random
  n, c        rows (points, tokens) and channels
  dtype       type of x and of what is computed from it
  clouds      clouds that the rows belong to
  groups, act norms: groups of channels, activation behind the norm (linear too)
  p           share that is dropped
  stream      drop: type of the residual stream
  scope       drop: what is dropped as one, "elements", "rows" or "clouds"
  form        quantise: 32 channels of a row share an exponent ("rows") or 32 rows of a channel ("columns")
  random      quantise: rounded at random, up with the probability of the remainder
  c_out       linear: output channels
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 32                       # elements that share an exponent in the 4-bit form
SITE = 5                         # which of a program's operators draws: part of the counter
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOW = 0xFFFFFFFF


def _case(name, op, n, c, dtype, **more):
    return dict({"op": op, "n": n, "c": c, "dtype": dtype}, **more, **({"name": name} if name else {}))


def listed():
    return [
        # a handful of points answered at once: launches and latency
        _case("norm_fwd_few", "norm_fwd", 3, 256, "bf16", clouds=1, groups=32, act="silu", p=0.0),
        # a training batch of eight outdoor clouds
        _case("norm_fwd_batch", "norm_fwd", 115_200, 64, "bf16", clouds=8, groups=8, act="gelu", p=0.1),
        # the gradients of an indoor cloud's layer in fp32, channels that fill no whole load
        _case("norm_bwd_ragged_f32", "norm_bwd", 99_991, 91, "f32", clouds=3, groups=13, act="silu", p=0.0),
        # the largest layer's: a million points, 256 channels
        _case("norm_bwd_large", "norm_bwd", 1_000_000, 256, "bf16", clouds=4, groups=32, act="silu", p=0.1),
        # the end of a branch on an fp32 residual stream, ragged
        _case("drop_fwd_ragged", "drop_fwd", 99_991, 91, "bf16", clouds=5, stream="f32", scope="elements", p=0.1),
        # its gradient in the largest layer
        _case("drop_bwd_large", "drop_bwd", 1_000_000, 256, "bf16", clouds=4, stream="bf16", scope="elements", p=0.25),
        # activations of a strided layer to 4 bits and back
        _case("quantise_rows", "quantise", 199_993, 128, "bf16", form="rows", random=False),
        # a gradient's columns, rounded at random, for the product that sums over the points
        _case("quantise_columns", "quantise", 100_000, 91, "f32", form="columns", random=True),
        # one token through a wide layer
        _case("linear_token", "linear", 1, 4096, "bf16", c_out=16_384, act="none"),
        # the widening half of a pointwise network on an outdoor scan
        _case("linear_points", "linear", 115_200, 64, "bf16", c_out=256, act="gelu"),
        # a large prompt or batch through a square layer
        _case("linear_large", "linear", 8192, 8192, "bf16", c_out=8192, act="none"),
        # gradients of a training step's pointwise layer: the weight's sums over all the points
        _case("linear_bwd_points", "linear_bwd", 200_000, 128, "bf16", c_out=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "drop_fwd", "drop_bwd", "quantise", "linear", "linear_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("linear", "linear_bwd"):
        c = rng.choice([32, 64, 128, 256, 512, _log_int(rng, 5, 8192)])
        c_out = rng.choice([32, 64, 128, 256, 512, _log_int(rng, 5, 16_384)])
        most = min((5e11 if op == "linear" else 2.5e11) / (c * c_out), 1.2e8 / max(c, c_out), 200_000)
        n = _log_int(rng, 1 if op == "linear" else 32, max(64, most))
        if op == "linear_bwd":
            return _case(None, op, n, c, dtype, c_out=c_out)
        return _case(None, op, n, c, dtype, c_out=c_out, act=rng.choice(["none", "relu", "silu", "gelu"]))
    c = rng.choice([32, 64, 128, 256, 512, rng.randint(5, 600)])
    n = _log_int(rng, 1, min(1_000_000, (200_000_000 if dtype == "bf16" else 100_000_000) // c))
    if op == "quantise":
        return _case(None, op, max(n, 20), c, dtype, form=rng.choice(["rows", "columns"]), random=rng.random() < 0.5)
    clouds = _log_int(rng, 1, min(64, n))
    p = rng.choice([0.0, 0.1, 0.25, 0.5])
    if op in ("norm_fwd", "norm_bwd"):
        groups = rng.choice([g for g in range(1, c + 1) if c % g == 0 and g <= 64])
        act = rng.choice(["none", "silu", "gelu"] + (["relu"] if op == "norm_fwd" else []))
        return _case(None, op, n, c, dtype, clouds=clouds, groups=groups, act=act, p=p)
    stream = "f32" if dtype == "f32" else rng.choice(["f32", "bf16"])
    return _case(None, op, n, c, dtype, clouds=clouds, stream=stream, scope=rng.choice(["elements", "elements", "rows", "clouds"]),
                 p=max(p, 0.05))


# ---- inputs ------------------------------------------------------------------------------------------------------

def _activations(g, n, c):
    """Rows of a network: channels of different scales and means, a few of them large."""
    scale = torch.exp(0.5 * torch.randn(c, generator=g, device="cuda"))
    scale = torch.where(torch.rand(c, generator=g, device="cuda") < 0.02, 10.0 * scale, scale)
    mean = 0.5 * scale * torch.randn(c, generator=g, device="cuda")
    return torch.randn(n, c, generator=g, device="cuda").mul_(scale).add_(mean)


def _offsets(g, n, clouds):
    """First row of every cloud, and n: clouds of different sizes."""
    share = torch.rand(clouds, generator=g, device="cuda", dtype=torch.float64) + 0.2
    cuts = (torch.cumsum(share, 0) / share.sum() * n).round().int()
    cuts[-1] = n
    return torch.cat([cuts.new_zeros(1), cuts])


def _affine(g, c):
    return 1.0 + 0.2 * torch.randn(c, generator=g, device="cuda"), 0.2 * torch.randn(c, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, n, c, dtype = case["op"], case["n"], case["c"], TYPES[case["dtype"]]
    s = {"case": case, "rng": torch.tensor([seed * 0x9E3779B97F4A7C1 % (1 << 62), 1000 + seed % 7], device="cuda")}
    if op in ("norm_fwd", "norm_bwd"):
        s["x"] = _activations(g, n, c).to(dtype)
        s["w"], s["b"] = _affine(g, c)
        s["offsets"] = _offsets(g, n, case["clouds"])
        s["bounds"] = s["offsets"].tolist()                                          # (for the plain form's loops over clouds)
        if op == "norm_bwd":
            s["dy"] = torch.randn(n, c, generator=g, device="cuda").to(dtype)
            s["mean_rstd"] = _statistics(s["x"], s["bounds"], case["groups"])       # the forward pass's
    elif op in ("drop_fwd", "drop_bwd"):
        s["offsets"] = _offsets(g, n, case["clouds"])
        if op == "drop_fwd":
            s["x"] = _activations(g, n, c).to(dtype)
            s["residual"] = _activations(g, n, c).to(TYPES[case["stream"]])
        else:
            s["dy"] = torch.randn(n, c, generator=g, device="cuda").to(TYPES[case["stream"]])
    elif op == "quantise":
        s["x"] = _activations(g, n, c).to(dtype)
    else:
        s["x"] = _activations(g, n, c).to(dtype)
        w = torch.randn(case["c_out"], c, generator=g, device="cuda") / math.sqrt(c)
        if op == "linear":
            s["q"], s["scales"] = _to_bits(w)
            s["bias"] = 0.2 * torch.randn(case["c_out"], generator=g, device="cuda")
        else:
            s["q"], s["scales"] = _to_bits(w.t().contiguous())
            s["dy"] = (torch.randn(n, case["c_out"], generator=g, device="cuda") / n).to(dtype)
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------

def _product32(a, b):
    """High and low words of products of 32-bit numbers held in 64 bits (which wrap; the words are right all the same)."""
    p = a * b
    return (p >> 32) & LOW, p & LOW


def _uniform16(rng, rows, c):
    """Random whole numbers 0 .. 65535 [rows, c]: ten rounds of Philox 4x32 (Salmon et al., "Parallel random numbers: as
    easy as 1, 2, 3", 2011) with the seed as key; the counter is (row * ceil(c / 8) + channel / 8, site, step); eight
    neighbouring channels take the sixteen-bit halves of the four words, low halves first."""
    blocks = -(-c // 8)
    seed, step = rng[0], rng[1]
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    x0 = torch.arange(rows * blocks, device="cuda", dtype=torch.int64)
    x1 = torch.full_like(x0, SITE)
    x2, x3 = (step & LOW).expand_as(x0), ((step >> 32) & LOW).expand_as(x0)
    for _ in range(10):
        h0, l0 = _product32(x0, 0xD2511F53)
        h1, l1 = _product32(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    words = torch.stack([x0, x1, x2, x3], 1)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).to(torch.int32)
    return halves.view(rows, 8 * blocks)[:, :c]


def _cloud_of(offsets, n):
    return torch.searchsorted(offsets[1:].contiguous(), torch.arange(n, device="cuda", dtype=torch.int32), right=True)


def _threshold(p):
    return int(math.floor(65536.0 * p + 0.5))


def _kept(s):
    """The factor of every element: 0, or what makes up for the share that is dropped; broadcast over rows or channels."""
    case = s["case"]
    n, c, scope = case["n"], case["c"], case.get("scope", "elements")
    t = _threshold(case["p"])
    if scope == "clouds":
        u = _uniform16(s["rng"], case["clouds"], 1)[_cloud_of(s["offsets"], n)]
    else:
        u = _uniform16(s["rng"], n, c if scope == "elements" else 1)
    return u >= t, 65536.0 / (65536 - t)


def _statistics(x, bounds, groups):
    """Mean and 1 / sqrt(variance + EPS) of every cloud and group, [clouds, groups, 2]."""
    out = []
    for a, b in zip(bounds[:-1], bounds[1:]):
        if a == b:
            out.append(torch.zeros(groups, 2, device="cuda"))
            continue
        v = x[a:b].double().view(b - a, groups, -1)
        mean = v.mean((0, 2))
        var = ((v - mean[None, :, None]) ** 2).mean((0, 2))
        out.append(torch.stack([mean, 1.0 / torch.sqrt(var + EPS)], 1).float())
    return torch.stack(out)


def _activate(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    if act == "silu":
        t = 1.0 / (1.0 + torch.exp(-z))
        return t * (1.0 + z * (1.0 - t))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return 1.0


def _plain_norm(s):
    case = s["case"]
    x, groups = s["x"].float(), case["groups"]
    n, c = x.shape
    width = c // groups
    stats = s["mean_rstd"] if case["op"] == "norm_bwd" else _statistics(s["x"], s["bounds"], groups)
    cloud = _cloud_of(s["offsets"], n)
    mean, rstd = (stats[:, :, i].repeat_interleave(width, 1)[cloud] for i in (0, 1))
    v = (x - mean) * rstd
    z = s["w"] * v + s["b"]
    if case["op"] == "norm_fwd":
        y = _activate(z, case["act"])
        if case["p"]:
            keep, factor = _kept(s)
            y = torch.where(keep, y * factor, 0.0)
        return {"y": y.to(s["x"].dtype), "mean_rstd": stats}
    dy = s["dy"].float()
    if case["p"]:
        keep, factor = _kept(s)
        dy = torch.where(keep, dy * factor, 0.0)
    dz = dy * _slope(z, case["act"])
    out = {"dw": (dz * v).double().sum(0).float(), "db": dz.double().sum(0).float()}
    d = s["w"] * dz
    dx = torch.empty_like(d)
    for a, b in zip(s["bounds"][:-1], s["bounds"][1:]):
        if a == b:
            continue
        dg, vg = d[a:b].view(b - a, groups, width), v[a:b].view(b - a, groups, width)
        m1 = dg.double().mean((0, 2), keepdim=True).float()
        m2 = (dg * vg).double().mean((0, 2), keepdim=True).float()
        dx[a:b] = (dg - m1 - vg * m2).view(b - a, c) * rstd[a:b]
    return dict(out, dx=dx.to(s["x"].dtype))


def _plain_drop(s):
    keep, factor = _kept(s)
    if s["case"]["op"] == "drop_fwd":
        return {"y": (s["residual"].float() + torch.where(keep, s["x"].float() * factor, 0.0)).to(s["residual"].dtype)}
    return {"dx": torch.where(keep, s["dy"].float() * factor, 0.0).to(TYPES[s["case"]["dtype"]])}


def _to_bits(x, u=None):
    """fp32 rows as 4-bit codes (sign, two bits of exponent, one of fraction), two a byte, the even channel's in the low half, and one
    power of two for 32 channels: the smallest with which nothing rounds past 6.  u: sixteen random bits each to round with."""
    n, c = x.shape
    blocks = -(-c // BLOCK)
    pad = (0, blocks * BLOCK - c)
    v = torch.nn.functional.pad(x, pad).view(n, blocks, BLOCK)
    amax = v.abs().amax(2)
    e = (((amax.view(torch.int32) + (0x200000 if u is None else 0x3FFFFF)) >> 23) - 2).clamp(1, 252)
    e = torch.where(torch.isfinite(amax), e, 255)
    a = v.abs() * ((254 - e.clamp(max=252)) << 23).view(torch.float32)[..., None]
    a = torch.where((e == 255)[..., None], 0.0, a)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    m = a / step
    if u is None:
        m = torch.round(m)
    else:
        low = torch.floor(m)
        up = ((m - low) * 65536.0).int() + torch.nn.functional.pad(u, pad).view(n, blocks, BLOCK) >= 65536
        m = low + up
    code = (m + torch.where(a < 2, 0.0, torch.where(a < 4, 2.0, 4.0))).clamp(max=7).to(torch.uint8)
    code = torch.where((e == 255)[..., None], 0, code + 8 * torch.signbit(v).to(torch.uint8)).to(torch.uint8).view(n, -1)
    scales = torch.zeros(n, 4 * (-(-c // 128)), dtype=torch.uint8, device=x.device)
    scales[:, :blocks] = e.to(torch.uint8)
    return code[:, 0::2] | code[:, 1::2] << 4, scales


def _values(q, scales, c):
    """What 4-bit rows stand for, in fp32."""
    code = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1)[:, :c].long()
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    table = torch.cat([table, -table])
    e = scales.int().repeat_interleave(BLOCK, 1)[:, :c]
    return torch.where(e == 255, math.nan, table[code] * (e << 23).view(torch.float32))


def _rounded(x, u=None, columns=False):
    if columns:
        return _values(*_to_bits(x.t().contiguous(), None if u is None else u.t()), x.shape[0])
    return _values(*_to_bits(x, u), x.shape[1])


def _plain_quantise(s):
    case = s["case"]
    u = _uniform16(s["rng"], case["n"], case["c"]) if case["random"] else None
    return {"values": _rounded(s["x"].float(), u, case["form"] == "columns").to(torch.bfloat16)}


def _plain_linear(s):
    case = s["case"]
    x, dtype = s["x"].float(), TYPES[case["dtype"]]
    if case["op"] == "linear":
        w = _values(s["q"], s["scales"], case["c"])
        return {"y": _activate(torch.matmul(_rounded(x), w.t()) + s["bias"], case["act"]).to(dtype)}
    w = _values(s["q"], s["scales"], case["c_out"])                                 # [c, c_out]
    u = _uniform16(s["rng"], case["n"], case["c_out"])
    dy = s["dy"].float()
    dx = torch.matmul(_rounded(dy, u), w.t())
    dw = torch.matmul(_rounded(dy, u, True), _rounded(x, None, True).t())
    return {"dx": dx.to(dtype), "dw": dw}


# ---- the framework's operators -----------------------------------------------------------------------------------

def _own(s):
    import paper_2511_23227_amd as pcpp

    case = s["case"]
    op, dtype = case["op"], TYPES[case["dtype"]]
    acts = {"none": pcpp.ACT_NONE, "relu": pcpp.ACT_RELU, "silu": pcpp.ACT_SILU, "gelu": pcpp.ACT_GELU}
    random = pcpp.Random(s["rng"], SITE)
    if op in ("norm_fwd", "norm_bwd"):
        how = dict(act=acts[case["act"]], p=case["p"], random=random)
        if op == "norm_fwd":
            y = pcpp.pcpp_group_norm_fwd(s["x"], case["groups"], s["w"], s["b"], s["offsets"], eps=EPS, **how)
            return {"y": y.y, "mean_rstd": y.mean_rstd}
        d = pcpp.pcpp_group_norm_bwd(s["dy"], s["x"], s["mean_rstd"], s["w"], s["b"], s["offsets"], **how)
        return {"dw": d.dw, "db": d.db, "dx": d.dx}
    if op in ("drop_fwd", "drop_bwd"):
        scope = {"elements": pcpp.DROP_ELEMENTS, "rows": pcpp.DROP_ROWS, "clouds": pcpp.DROP_CLOUDS}[case["scope"]]
        how = dict(scope=scope, offsets=s["offsets"] if case["scope"] == "clouds" else None)
        if op == "drop_fwd":
            return {"y": pcpp.pcpp_dropout_fwd(s["x"], case["p"], random, s["residual"], **how)}
        return {"dx": pcpp.pcpp_dropout_bwd(s["dy"], case["p"], random, dtype=dtype, **how)}
    if op == "quantise":
        columns = case["form"] == "columns"
        m = pcpp.pcpp_mx_pack(s["x"], rows=not columns, columns=columns, random=random if case["random"] else None)
        return {"values": pcpp.pcpp_mx_unpack(m.columns if columns else m.rows)}
    if op == "linear":
        return {"y": pcpp.pcpp_mx_linear(s["x"], pcpp.MxRows(s["q"], s["scales"], case["c"]), s["bias"], act=acts[case["act"]])}
    dy = pcpp.pcpp_mx_pack(s["dy"], columns=True, random=random)
    x = pcpp.pcpp_mx_pack(s["x"], rows=False, columns=True)
    return {"dx": pcpp.pcpp_mx_product(dy.rows, pcpp.MxRows(s["q"], s["scales"], case["c_out"]), dtype=dtype),
            "dw": pcpp.pcpp_mx_product(dy.columns, x.columns, dtype=torch.float32)}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return {"norm_fwd": _plain_norm, "norm_bwd": _plain_norm, "drop_fwd": _plain_drop, "drop_bwd": _plain_drop,
            "quantise": _plain_quantise, "linear": _plain_linear, "linear_bwd": _plain_linear}[op](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    op, n, c = case["op"], case["n"], case["c"]
    size = {"f32": 4, "bf16": 2}
    es = size[case["dtype"]]
    bits = lambda rows, k: rows * (k / 2 + k / BLOCK)  # noqa: E731
    if op == "norm_fwd":
        return {"bytes": 2 * n * c * es + 8 * c + 8 * case["clouds"] * case["groups"], "flops": 12 * n * c}
    if op == "norm_bwd":
        return {"bytes": 3 * n * c * es + 16 * c + 8 * case["clouds"] * case["groups"], "flops": 28 * n * c}
    if op == "drop_fwd":
        return {"bytes": n * c * (es + 2 * size[case["stream"]]), "flops": 2 * n * c}
    if op == "drop_bwd":
        return {"bytes": n * c * (es + size[case["stream"]]), "flops": n * c}
    if op == "quantise":
        return {"bytes": n * c * (es + 2) + bits(n, c), "flops": 2 * n * c}
    m = case["c_out"]
    if op == "linear":
        return {"bytes": n * c * es + bits(m, c) + 4 * m + n * m * es, "flops": 2 * n * c * m}
    return {"bytes": 2 * n * c * es + n * m * es + bits(m, c) + 4 * m * c, "flops": 4 * n * c * m}


# ---- in 64 bits --------------------------------------------------------------------------------------------------

def _exact_draws(rng, rows, c):
    """The random numbers by way of products of 16-bit halves, the counter and the key as four columns."""
    groups = (c + 7) // 8
    seed, step = (int(v) & 0xFFFFFFFFFFFFFFFF for v in rng.tolist())
    x = [torch.arange(rows * groups, device="cuda"), SITE, step % 2 ** 32, step // 2 ** 32]
    x = [x[0]] + [torch.full_like(x[0], v) for v in x[1:]]

    def times(v, by):
        lo, hi = v % 65536, v // 65536
        bl, bh = by % 65536, by // 65536
        low, mid = lo * bl, lo * bh + hi * bl                      # below 2^33
        low = low + mid % 65536 * 65536
        return hi * bh + mid // 65536 + low // 2 ** 32, low % 2 ** 32

    key = [seed % 2 ** 32, seed // 2 ** 32]
    for _ in range(10):
        a, b = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
        x = [torch.bitwise_xor(torch.bitwise_xor(b[0], x[1]), key[0]), b[1],
             torch.bitwise_xor(torch.bitwise_xor(a[0], x[3]), key[1]), a[1]]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    out = torch.empty(rows * groups, 8, dtype=torch.int32, device="cuda")
    for i in range(4):
        out[:, 2 * i], out[:, 2 * i + 1] = x[i] % 65536, x[i] // 65536
    return out.view(rows, -1)[:, :c]


def _exact_factor(case, s):
    t = round(case["p"] * 65536)                                   # (none of these is half of one)
    n = case["n"]
    scope = case.get("scope", "elements")
    if scope == "clouds":
        u = _exact_draws(s["rng"], case["clouds"], 1).repeat_interleave((s["offsets"][1:] - s["offsets"][:-1]).long(), 0)
    else:
        u = _exact_draws(s["rng"], n, case["c"] if scope == "elements" else 1)
    return (u >= t).double() * (65536 / (65536 - t))


def _power(p):
    """2^p in 64 bits (torch's ldexp takes powers of two that 32 bits round)."""
    return ((p.long() + 1023) << 52).view(torch.float64)


def _exact_round(x, u=None):
    """4-bit values of rows in 64 bits."""
    n, c = x.shape
    padded = x.new_zeros(n, -(-c // BLOCK) * BLOCK)
    padded[:, :c] = x
    v = padded.reshape(n, -1, BLOCK)
    amax = v.abs().amax(2, keepdim=True)
    p = torch.frexp(amax).exponent - 3                             # amax in [4, 8) steps
    top = amax * _power(-p)
    p = torch.where(top >= 7 if u is None else top > 6, p + 1, p).clamp(-126, 125)
    a = v * _power(-p)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    below = torch.searchsorted(grid, a.abs().contiguous(), right=True) - 1
    above = (below + 1).clamp(max=7)
    lo, hi = grid[below], grid[above]
    gap = torch.where(hi > lo, hi - lo, 1.0)
    rest = (a.abs() - lo) / gap
    if u is None:
        up = (rest > 0.5) | ((rest == 0.5) & (below % 2 == 1))
    else:
        w = torch.zeros(n, padded.shape[1], dtype=torch.float64, device="cuda")
        w[:, :c] = u
        up = torch.floor(rest * 65536) + w.reshape(v.shape) >= 65536
    r = torch.copysign(torch.where(up, hi, lo), a) * _power(p)
    return r.reshape(n, -1)[:, :c]


def _exact_values(q, scales, c):
    n = q.shape[0]
    code = torch.empty(n, 2 * q.shape[1], dtype=torch.int64, device="cuda")
    code[:, 0::2], code[:, 1::2] = (q % 16).long(), (q // 16).long()
    exponent, fraction, sign = code // 2 % 4, code % 2, code // 8
    v = torch.where(exponent == 0, 0.5 * fraction.double(), (1.0 + 0.5 * fraction.double()) * _power(exponent - 1))
    v = (1 - 2 * sign) * v
    block = torch.arange(c, device="cuda") // BLOCK
    return v[:, :c] * _power(scales[:, block].int() - 127)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "drop_fwd":
        return {"y": s["residual"].double() + s["x"].double() * _exact_factor(case, s)}
    if op == "drop_bwd":
        return {"dx": s["dy"].double() * _exact_factor(case, s)}
    if op == "quantise":
        u = _exact_draws(s["rng"], case["n"], case["c"]).double() if case["random"] else None
        x = s["x"].double()
        if case["form"] == "columns":
            x, u = x.t(), None if u is None else u.t()
        return {"values": _exact_round(x, u)}
    act = {"none": lambda z: z, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[case.get("act", "none")]
    if op == "linear":
        y = _exact_round(s["x"].double()) @ _exact_values(s["q"], s["scales"], case["c"]).T
        return {"y": act(y + s["bias"].double())}
    if op == "linear_bwd":
        dy, u = s["dy"].double(), _exact_draws(s["rng"], case["n"], case["c_out"]).double()
        return {"dx": _exact_round(dy, u) @ _exact_values(s["q"], s["scales"], case["c_out"]).T,
                "dw": _exact_round(dy.t(), u.t()) @ _exact_round(s["x"].double().t()).T}
    # norms: cloud by cloud, the gradients by way of automatic differentiation
    train = op == "norm_bwd"
    groups = case["groups"]
    w, b = s["w"].double().requires_grad_(train), s["b"].double().requires_grad_(train)
    factor = _exact_factor(case, s) if case["p"] else None
    ys, stats, dxs = [], [], []
    dw, db = torch.zeros_like(s["w"], dtype=torch.float64), torch.zeros_like(s["b"], dtype=torch.float64)
    for lo, hi in zip(s["bounds"][:-1], s["bounds"][1:]):
        if lo == hi:
            stats.append(torch.zeros(groups, 2, dtype=torch.float64, device="cuda"))
            continue
        x = s["x"][lo:hi].double().requires_grad_(train)
        v = x.view(hi - lo, groups, -1)
        var, mean = torch.var_mean(v, (0, 2), correction=0)
        rstd = torch.rsqrt(var + EPS)
        y = act(((v - mean[:, None]) * rstd[:, None]).view(hi - lo, -1) * w + b)
        if factor is not None:
            y = y * factor[lo:hi]
        if train:
            got = torch.autograd.grad(y, [x, w, b], s["dy"][lo:hi].double())
            dxs.append(got[0])
            dw, db = dw + got[1], db + got[2]
        else:
            ys.append(y)
            stats.append(torch.stack([mean, rstd], 1))
    if train:
        return {"dw": dw, "db": db, "dx": torch.cat(dxs)}
    return {"y": torch.cat(ys), "mean_rstd": torch.stack(stats)}
