"""The operators around a convolution in a training step, and in an answer, as measurable cases: the norms, gate and
residual between two blocks, activations kept in 8 bits with the gradients that read them, and the log probabilities of
a head's classes with their gradient.

A case is a dict of plain values:
  op          block_fwd  residual, gate and post norm of a block with the pre norm of the next one
              block_bwd  their gradients
              pack       activations to 8 bits and back
              weight     weight gradient of a convolution whose input was kept in 8 bits
              answer     log probability of a label, entropy and most probable alternatives of every row
              loss       log probability and entropy of every row and the gradient of the logits
  n, c        rows (points, tokens) and channels, or classes for `answer` and `loss`
  dtype       type of the block's tensors, of the packed activations' source, of the logits
  stream      block: type of the residual stream
  norm, gate  block: kind of both norms; columns of the gate's logits, "none", "row" or "full"
  packed      block: forward, the block's output and the next block's input are written in 8 bits too; backward, the
              block's output is read from 8 bits
  c_out, t, neighbours, layer     weight: output channels, cells per axis, mean inputs per output, outputs at the inputs
              ("same") or at a quarter of them ("down")
  top         answer: alternatives
  mask        answer, loss: share of the classes that are masked (half with -inf, half with the type's lowest)
"""
import math

import torch

own = False

RADIUS = 0.05                    # of a neighbourhood, metres
EPS = 1e-6
BLOCK = 32                       # channels that share an exponent in the 8-bit form
PIECE = 1024                     # triplets that the plain weight gradient takes at a time
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _block(name, op, n, c, dtype, stream, norm="rms", gate="full", packed=False):
    return dict({"op": op, "n": n, "c": c, "dtype": dtype, "stream": stream, "norm": norm, "gate": gate, "packed": packed},
                **({"name": name} if name else {}))


def _pack_case(name, n, c, dtype):
    return dict({"op": "pack", "n": n, "c": c, "dtype": dtype}, **({"name": name} if name else {}))


def _weight(name, n, c, c_out, dtype, t, neighbours, layer="same"):
    return dict({"op": "weight", "n": n, "c": c, "c_out": c_out, "dtype": dtype, "t": t, "neighbours": neighbours,
                 "layer": layer}, **({"name": name} if name else {}))


def _head(name, op, n, c, dtype, top=0, mask=0.0):
    return dict({"op": op, "n": n, "c": c, "dtype": dtype, "top": top, "mask": mask}, **({"name": name} if name else {}))


def listed():
    return [
        # a handful of rows answered at once: launches and latency
        _block("block_fwd_few", "block_fwd", 3, 256, "bf16", "bf16"),
        # between two layers of an indoor network in fp32, inference
        _block("block_fwd_indoor_f32", "block_fwd", 100_000, 32, "f32", "f32", norm="layer", gate="row"),
        # an outdoor network's training step with an fp32 residual stream: what the backward pass reads is kept in 8 bits
        _block("block_fwd_train", "block_fwd", 115_200, 64, "bf16", "f32", packed=True),
        # its backward pass; channels that fill no whole load
        _block("block_bwd_ragged", "block_bwd", 99_991, 91, "bf16", "f32", norm="layer", gate="row", packed=True),
        # the largest layer's: a million points, 256 channels
        _block("block_bwd_large", "block_bwd", 1_000_000, 256, "bf16", "bf16"),
        # activations of a strided layer to 8 bits and back
        _pack_case("pack_strided", 199_993, 128, "bf16"),
        # a small fp32 cloud's, ragged
        _pack_case("pack_small_f32", 2048, 20, "f32"),
        # weight gradient of an early indoor layer in fp32
        _weight("weight_indoor_f32", 100_000, 32, 32, "f32", 3, 24.3),
        # of the strided layer that doubles the channels
        _weight("weight_strided_bf16", 200_000, 64, 128, "bf16", 3, 92.0, "down"),
        # a class for every point of a scan, with the runners-up
        _head("answer_points", "answer", 115_200, 17, "f32", top=3),
        # one token out of a large vocabulary of which a grammar allows two thirds, with the alternatives
        _head("answer_token", "answer", 1, 131_072, "bf16", top=20, mask=0.3),
        # a training batch over a vocabulary
        _head("loss_vocabulary", "loss", 4096, 32_768, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["block_fwd", "block_bwd", "pack", "weight", "answer", "loss"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op in ("block_fwd", "block_bwd"):
        c = rng.choice([32, 64, 128, 256, 512, rng.randint(5, 600)])
        n = _log_int(rng, 1, min(1_000_000, (200_000_000 if dtype == "bf16" else 100_000_000) // c))
        stream = "f32" if dtype == "f32" else rng.choice(["f32", "bf16"])
        return _block(None, op, n, c, dtype, stream, rng.choice(["rms", "rms", "layer"]), rng.choice(["none", "row", "full"]),
                      rng.random() < 0.5)
    if op == "pack":
        c = rng.choice([32, 64, 128, 256, rng.randint(5, 600)])
        return _pack_case(None, _log_int(rng, 100, min(1_000_000, 200_000_000 // c)), c, dtype)
    if op == "weight":
        if rng.random() < 0.75:
            c, c_out = rng.choice([(16, 32), (32, 32), (32, 64), (64, 64), (64, 128), (128, 128), (128, 64), (256, 256)])
        else:
            c, c_out = rng.randint(5, 130), rng.randint(6, 130)
        neighbours = round(math.exp(rng.uniform(math.log(8.0), math.log(92.0))), 1)
        most = 36e9 / (c * c_out * (4.0 if dtype == "f32" else 1.0)) / neighbours
        n = _log_int(rng, 2_000, max(2_001, min(200_000, most)))
        return _weight(None, n, c, c_out, dtype, rng.choice([2, 3, 3, 4]), neighbours, rng.choice(["same", "down"]))
    c = _log_int(rng, 2, 131_072)
    n = _log_int(rng, 1, max(1, min(1_000_000, 100_000_000 // c)))
    if op == "answer":
        return _head(None, op, n, c, dtype, min(c, rng.choice([0, 1, 3, 5, 20])), rng.choice([0.0, 0.0, 0.3]))
    return _head(None, op, n, c, dtype, 0, rng.choice([0.0, 0.0, 0.3]))


# ---- inputs ------------------------------------------------------------------------------------------------------

def _activations(g, n, c, zeros=0.0):
    """Rows of a network: channels of different scales, a few of them large, and a share of rows that are zero."""
    scale = torch.exp(0.5 * torch.randn(c, generator=g, device="cuda"))
    scale = torch.where(torch.rand(c, generator=g, device="cuda") < 0.02, 10.0 * scale, scale)
    rows = torch.rand(n, 1, generator=g, device="cuda") >= zeros
    return torch.randn(n, c, generator=g, device="cuda") * scale * rows


def _surface(g, n, neighbours):
    """Points on noisy rectangles of a room, in random order: about `neighbours` of them within RADIUS of each."""
    planes = 40
    side = math.sqrt(n * math.pi * RADIUS ** 2 / neighbours / planes)
    axis = torch.randint(3, (planes,), generator=g, device="cuda")
    corner = torch.rand(planes, 3, generator=g, device="cuda") * max(4.0, 4.0 * side)
    which = torch.randint(planes, (n,), generator=g, device="cuda")
    at = torch.rand(n, 3, generator=g, device="cuda") * side
    at = at * (torch.arange(3, device="cuda") != axis[which][:, None])
    return corner[which] + at + 0.005 * torch.randn(n, 3, generator=g, device="cuda")


def _triplets(points, centres, t):
    """All (o, i, k) with i within RADIUS of o, k the cell of the offset, in ascending (k, o, i) order; run starts by k."""
    p, q = points.double(), centres.double()
    low = p.min(0).values - 2 * RADIUS
    cell, home = ((p - low) / RADIUS).floor().long(), ((q - low) / RADIUS).floor().long()
    size = cell.max(0).values + 3
    number = lambda v: (v[..., 0] * size[1] + v[..., 1]) * size[2] + v[..., 2]  # noqa: E731
    order = torch.sort(number(cell)).indices
    sorted_cells = number(cell)[order]
    step = torch.arange(-1, 2, device="cuda")
    stencil = torch.cartesian_prod(step, step, step)
    wanted = number(home[:, None] + stencil).reshape(-1)
    first = torch.searchsorted(sorted_cells, wanted)
    count = torch.searchsorted(sorted_cells, wanted, right=True) - first
    o = torch.repeat_interleave(torch.arange(len(q), device="cuda").repeat_interleave(len(stencil)), count)
    start = torch.repeat_interleave(first - (torch.cumsum(count, 0) - count), count)
    i = order[start + torch.arange(len(o), device="cuda")]
    d = p[i] - q[o]
    near = (d * d).sum(1) <= RADIUS ** 2
    o, i, d = o[near], i[near], d[near]
    k = ((d + RADIUS) * (t / (2 * RADIUS))).floor().long().clamp(0, t - 1)
    k = (k[:, 0] * t + k[:, 1]) * t + k[:, 2]
    order = torch.sort((k * len(q) + o) * len(p) + i).indices
    o, i, k = o[order].int(), i[order].int(), k[order].int()
    seg = torch.searchsorted(k, torch.arange(t ** 3 + 1, device="cuda", dtype=torch.int32))
    return o, i, k, seg


def _logits(g, case):
    x = 2.5 * torch.randn(case["n"], case["c"], generator=g, device="cuda") + 3.0 * torch.randn(case["n"], 1, generator=g, device="cuda")
    x = x.to(TYPES[case["dtype"]])
    if case["mask"]:
        u = torch.rand(case["c"], generator=g, device="cuda")
        x = torch.where(u < 0.5 * case["mask"], -math.inf, x)
        x = torch.where((u >= 0.5 * case["mask"]) & (u < case["mask"]), torch.finfo(x.dtype).min, x)
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, n, c, dtype = case["op"], case["n"], case["c"], TYPES[case["dtype"]]
    s = {"case": case}
    if op in ("block_fwd", "block_bwd"):
        f = _activations(g, n, c).to(dtype)
        if case["packed"] and op == "block_bwd":
            s["q"], s["e"] = _pack(f.float())
        else:
            s["f"] = f
        if case["gate"] != "none":
            s["gate"] = torch.randn(n, c if case["gate"] == "full" else 1, generator=g, device="cuda").to(dtype)
        s["w_post"] = 1.0 + 0.2 * torch.randn(c, generator=g, device="cuda")
        s["w_pre"] = 1.0 + 0.2 * torch.randn(c, generator=g, device="cuda")
        # forward: the residual stream before the block; backward: behind it
        s["x"] = _activations(g, n, c).to(TYPES[case["stream"]])
        if op == "block_bwd":
            s["dr"] = torch.randn(n, c, generator=g, device="cuda").to(TYPES[case["stream"]])
            s["dh"] = torch.randn(n, c, generator=g, device="cuda").to(dtype)
    elif op == "pack":
        s["x"] = _activations(g, n, c, 0.002).to(dtype)
    elif op == "weight":
        points = _surface(g, n, case["neighbours"])
        centres = points[: max(1, n // 4)].contiguous() if case["layer"] == "down" else points
        s["tri_o"], s["tri_i"], s["tri_k"], s["seg"] = _triplets(points, centres, case["t"])
        s["q"], s["e"] = _pack(_activations(g, n, c, 0.002).to(dtype).float())
        s["dy"] = torch.randn(len(centres), case["c_out"], generator=g, device="cuda").to(dtype)
        pieces = -(-(s["seg"][1:] - s["seg"][:-1]) // PIECE)
        s["cell"] = torch.repeat_interleave(torch.arange(len(pieces), device="cuda"), pieces)
        nth = torch.arange(len(s["cell"]), device="cuda") - (torch.cumsum(pieces, 0) - pieces)[s["cell"]]
        s["piece"] = s["seg"][s["cell"]] + PIECE * nth
    else:
        s["x"] = _logits(g, case)
        s["labels"] = torch.randint(c, (n,), generator=g, device="cuda", dtype=torch.int32)
        s["labels"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.02, -1, s["labels"])   # rows without a label
        s["d_log_prob"] = -torch.rand(n, generator=g, device="cuda") / n
        s["d_entropy"] = 0.01 * torch.rand(n, generator=g, device="cuda") / n
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------

def _pack(x):
    """fp32 rows as int8 and one exponent for 32 channels: value = q 2^(e - 127), 255 where a value is not finite."""
    n, c = x.shape
    blocks = -(-c // BLOCK)
    v = torch.nn.functional.pad(x, (0, blocks * BLOCK - c)).view(n, blocks, BLOCK)
    amax = v.abs().amax(2)
    fine = torch.isfinite(amax)
    e = torch.where(fine, (((amax.view(torch.int32) + 0x10000) >> 23) - 6).clamp(min=1), 255)
    scale = ((254 - e) << 23).view(torch.float32)
    q = torch.round(torch.where(fine[..., None], v * scale[..., None], 0.0))
    codes = torch.zeros(n, 4 * (-(-c // 128)), dtype=torch.uint8, device=x.device)
    codes[:, :blocks] = e.to(torch.uint8)
    return q.view(n, -1)[:, :c].to(torch.int8).contiguous(), codes


def _unpack(q, codes):
    e = codes.int().repeat_interleave(BLOCK, 1)[:, : q.shape[1]]
    return torch.where(e == 255, math.nan, q.float() * (e << 23).view(torch.float32))


def _norm(v, kind):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * rstd, rstd


def _norm_bwd(y, v, rstd, kind):
    d = y - v * (y * v).mean(1, keepdim=True)
    if kind == "layer":
        d = d - y.mean(1, keepdim=True)
    return d * rstd


def _sigmoid(s):
    return 1.0 / (1.0 + torch.exp(-s["gate"].float())) if "gate" in s else 1.0


def _residual_scale(case):
    return 0.75 if case["norm"] == "rms" else 1.0


def _plain_block_fwd(s):
    case = s["case"]
    f, dtype = s["f"].float(), TYPES[case["dtype"]]
    r = _residual_scale(case) * s["x"].float() + _sigmoid(s) * (s["w_post"] * _norm(f, case["norm"])[0])
    h = s["w_pre"] * _norm(r, case["norm"])[0]
    out = {"r": r.to(TYPES[case["stream"]]), "h": h.to(dtype)}
    if case["packed"]:
        out["f8"], out["h8"] = _unpack(*_pack(f)).to(torch.bfloat16), _unpack(*_pack(h)).to(torch.bfloat16)
    return out


def _plain_block_bwd(s):
    case = s["case"]
    kind, dtype, stream = case["norm"], TYPES[case["dtype"]], TYPES[case["stream"]]
    f = _unpack(s["q"], s["e"]) if case["packed"] else s["f"].float()
    dh, sigma = s["dh"].float(), _sigmoid(s)
    nr, rstd_r = _norm(s["x"].float(), kind)
    nf, rstd_f = _norm(f, kind)
    d = s["dr"].float() + _norm_bwd(s["w_pre"] * dh, nr, rstd_r, kind)
    du = d * sigma
    out = {"dx": (_residual_scale(case) * d).to(stream), "df": _norm_bwd(s["w_post"] * du, nf, rstd_f, kind).to(dtype),
           "dw_post": (du * nf).sum(0), "dw_pre": (dh * nr).sum(0)}
    if case["gate"] != "none":
        dg = du * (1.0 - sigma) * (s["w_post"] * nf)
        out["dgate"] = (dg if case["gate"] == "full" else dg.sum(1, keepdim=True)).to(dtype)
    return out


def _plain_weight(s):
    # the cells' runs in pieces of PIECE triplets, the last one of a cell filled up; one batched product, summed by cell
    row = s["piece"][:, None] + torch.arange(PIECE, device="cuda")
    inside = row < s["seg"][1:][s["cell"]][:, None]
    row = row.clamp(max=len(s["tri_o"]) - 1)
    x = _unpack(s["q"], s["e"])[s["tri_i"][row].long()]
    dy = s["dy"].float()[s["tri_o"][row].long()] * inside[..., None]
    dw = torch.zeros(len(s["seg"]) - 1, dy.shape[2], x.shape[2], device="cuda")
    return {"dw": dw.index_add_(0, s["cell"], torch.matmul(dy.transpose(1, 2).contiguous(), x))}


def _plain_head(s):
    x, labels = s["x"].float(), s["labels"].long()
    m = x.amax(1, keepdim=True)
    z = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    total = z.sum(1, keepdim=True)                     # 0: every class of the row is masked
    lp = torch.where(total > 0, x - (m + torch.log(total)), -math.inf)
    p = torch.where(total > 0, z / total, 0.0)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    given = (labels >= 0)[:, None]
    log_prob = torch.where(given, torch.gather(lp, 1, labels.clamp(min=0)[:, None]), 0.0)[:, 0]
    return x, labels, p, lp, entropy, given, log_prob


def _plain_answer(s):
    x, _, _, lp, entropy, _, log_prob = _plain_head(s)
    out = {"log_prob": log_prob, "entropy": entropy}
    if s["case"]["top"]:
        index = torch.sort(x, dim=1, descending=True, stable=True).indices[:, : s["case"]["top"]]
        out["top_log_prob"], out["top_index"] = torch.gather(lp, 1, index), index.int()
    return out


def _plain_loss(s):
    x, labels, p, lp, entropy, given, log_prob = _plain_head(s)
    hit = (torch.arange(x.shape[1], device=x.device) == labels[:, None]).float()
    d = torch.where(given, s["d_log_prob"][:, None] * (hit - p), 0.0)
    d = d - s["d_entropy"][:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
    return {"log_prob": log_prob, "entropy": entropy, "d_logits": d.to(s["x"].dtype)}


# ---- the framework's operators -----------------------------------------------------------------------------------

def _own(s):
    import paper_2511_23227_amd as pcpp

    case = s["case"]
    op = case["op"]
    if op in ("block_fwd", "block_bwd"):
        kind = pcpp.NORM_LAYER if case["norm"] == "layer" else pcpp.NORM_RMS
        how = dict(post_norm=kind, pre_norm=kind, residual_scale=_residual_scale(case), eps=EPS)
        if op == "block_fwd":
            y = pcpp.pcpp_block_norm_fwd(s["x"], s["f"], s.get("gate"), s["w_post"], s["w_pre"], pack_f=case["packed"],
                                         pack_h=case["packed"], **how)
            out = {"r": y.r, "h": y.h}
            if case["packed"]:
                out["f8"], out["h8"] = pcpp.pcpp_act_unpack(y.f_packed), pcpp.pcpp_act_unpack(y.h_packed)
            return out
        f = pcpp.Packed(s["q"], s["e"]) if case["packed"] else s["f"]
        y = pcpp.pcpp_block_norm_bwd(s["dr"], s["dh"], s["x"], f, s.get("gate"), s["w_post"], s["w_pre"], **how)
        out = {"dx": y.dx, "df": y.df, "dw_post": y.dw_post, "dw_pre": y.dw_pre}
        return dict(out, dgate=y.dgate) if case["gate"] != "none" else out
    if op == "pack":
        return {"values": pcpp.pcpp_act_unpack(pcpp.pcpp_act_pack(s["x"]))}
    if op == "weight":
        T = pcpp.Triplets(s["tri_o"], s["tri_i"], s["tri_k"], s["seg"], s["tri_o"].numel(), s["q"].shape[0], s["dy"].shape[0],
                          case["t"], None, 0)
        return {"dw": pcpp.pcpp_mvmr_bwd_weight_packed(pcpp.Packed(s["q"], s["e"]), s["dy"], T)}
    y = pcpp.pcpp_log_probs_fwd(s["x"], s["labels"], n_top=case["top"])
    out = {"log_prob": y.log_prob, "entropy": y.entropy}
    if op == "answer":
        return dict(out, top_log_prob=y.top_log_prob, top_index=y.top_index) if case["top"] else out
    return dict(out, d_logits=pcpp.pcpp_log_probs_bwd(s["x"], s["labels"], y, s["d_log_prob"], s["d_entropy"]))


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "pack":
        return {"values": _unpack(*_pack(state["x"].float())).to(torch.bfloat16)}
    return {"block_fwd": _plain_block_fwd, "block_bwd": _plain_block_bwd, "weight": _plain_weight, "answer": _plain_answer,
            "loss": _plain_loss}[op](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    op, n, c = case["op"], case["n"], case["c"]
    size = {"f32": 4, "bf16": 2}
    es = size[case["dtype"]]
    packed = c + -(-c // BLOCK)                        # bytes of a row in 8 bits
    if op in ("block_fwd", "block_bwd"):
        ss = size[case["stream"]]
        gate = {"none": 0, "row": 1, "full": c}[case["gate"]] * es
        if op == "block_fwd":
            row = 2 * c * ss + 2 * c * es + gate + (2 * (packed + 2 * c) if case["packed"] else 0)
            return {"bytes": n * row + 8 * c, "flops": 14 * n * c}
        row = 3 * c * ss + (2 * c * es + packed if case["packed"] else 3 * c * es) + 2 * gate
        return {"bytes": n * row + 16 * c, "flops": 26 * n * c}
    if op == "pack":
        return {"bytes": n * (c * es + packed + 2 * c), "flops": 4 * n * c}
    if op == "weight":
        n_out, k = (n // 4 if case["layer"] == "down" else n), case["t"] ** 3
        pairs = n_out * case["neighbours"]
        return {"bytes": n * packed + n_out * case["c_out"] * es + 8 * pairs + 4 * k * c * case["c_out"],
                "flops": 2 * pairs * c * case["c_out"]}
    if op == "answer":
        return {"bytes": n * (c * es + 12 + 8 * case["top"]), "flops": 6 * n * c}
    return {"bytes": n * (2 * c * es + 20), "flops": 14 * n * c}


# ---- in 64 bits --------------------------------------------------------------------------------------------------

def _exact_values(q, codes):
    c = q.shape[1]
    channel = torch.arange(c, device=q.device) // BLOCK
    code = codes[:, channel].double()
    return torch.ldexp(q.double(), code - 127.0)


def _exact_round(x):
    """8-bit values of rows in 64 bits: the smallest power of two with which no value of 32 channels rounds past 127."""
    n, c = x.shape
    padded = x.new_zeros(n, -(-c // BLOCK) * BLOCK)
    padded[:, :c] = x
    v = padded.reshape(n, -1, BLOCK)
    amax = v.abs().amax(2, keepdim=True)
    p = torch.frexp(amax).exponent - 7                 # amax in [64, 128) steps
    p = torch.where(torch.round(torch.ldexp(amax, -p)) > 127, p + 1, p).clamp(min=-126)
    return torch.ldexp(torch.round(torch.ldexp(v, -p)), p).reshape(n, -1)[:, :c]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pack":
        return {"values": _exact_round(s["x"].double())}
    if op == "weight":
        x, dy = _exact_values(s["q"], s["e"]), s["dy"].double()
        seg, dw = s["seg"].tolist(), []
        for a, b in zip(seg[:-1], seg[1:]):
            dw.append(dy[s["tri_o"][a:b].long()].T @ x[s["tri_i"][a:b].long()])
        return {"dw": torch.stack(dw)}
    if op in ("answer", "loss"):
        x, labels = s["x"].double(), s["labels"].long()
        lp = torch.log_softmax(x, 1)
        lp = torch.where((x > -math.inf).any(1, keepdim=True), lp, -math.inf)
        p = lp.exp()
        plogp = torch.where(p > 0, p * lp, 0.0)
        h = -plogp.sum(1)
        rows = torch.arange(len(x), device=x.device)
        given = (labels >= 0).double()
        picked = lp[rows, labels.clamp(min=0)]
        out = {"log_prob": torch.where(labels >= 0, picked, 0.0), "entropy": h}
        if op == "answer":
            if case["top"]:
                index = torch.sort(-x, dim=1, stable=True).indices[:, : case["top"]]
                out["top_log_prob"], out["top_index"] = lp[rows[:, None], index], index.int()
            return out
        d = -p * (given * s["d_log_prob"].double())[:, None]
        d[rows, labels.clamp(min=0)] += given * s["d_log_prob"].double()
        return dict(out, d_logits=d - s["d_entropy"].double()[:, None] * (plogp + p * h[:, None]))
    # a block: its gradients by way of automatic differentiation
    train = op == "block_bwd"
    f = _exact_values(s["q"], s["e"]) if "q" in s else s["f"].double()
    scale = _residual_scale(case)
    ins = {"x": s["x"].double(), "f": f, "w_post": s["w_post"].double(), "w_pre": s["w_pre"].double()}
    if "gate" in s:
        ins["gate"] = s["gate"].double()
    for v in ins.values():
        v.requires_grad_(train)

    def norm(v):
        if case["norm"] == "layer":
            v = v - v.mean(1, keepdim=True)
        return v * torch.rsqrt(v.pow(2).mean(1, keepdim=True) + EPS)

    branch = norm(ins["f"]) * ins["w_post"]
    if "gate" in ins:
        branch = torch.sigmoid(ins["gate"]) * branch
    if not train:
        r = scale * ins["x"] + branch
        h = norm(r) * ins["w_pre"]
        out = {"r": r, "h": h}
        return dict(out, f8=_exact_round(f), h8=_exact_round(h)) if case["packed"] else out
    # the stream behind the block is given (s["x"]); what flows to it goes on to the stream before and to the branch
    h = norm(ins["x"]) * ins["w_pre"]
    to_r, dw_pre = torch.autograd.grad(h, [ins["x"], ins["w_pre"]], s["dh"].double())
    d = s["dr"].double() + to_r
    names = [k for k in ("f", "w_post", "gate") if k in ins]
    got = dict(zip(names, torch.autograd.grad(branch, [ins[k] for k in names], d)))
    out = {"dx": scale * d, "df": got["f"], "dw_post": got["w_post"], "dw_pre": dw_pre}
    return dict(out, dgate=got["gate"]) if "gate" in got else out
