"""The operators around the convolution against plain 64-bit forms: activations in 8 bits and the weight gradient that reads
them, norms with gate and residual, log probabilities; and their gradients against differences.

Tolerances.  u = 2^-24 is the rounding of fp32.  A sum of c terms is off by at most c u times the sum of the terms' magnitudes, so
every fp32 result is held to 8 (c + 40) u times the magnitude that the formula's terms reach (the references carry it along); a result
in bf16 (eight significant bits) may be off by its own rounding, 2^-8 of it, too.  What has no rounding (8-bit values, indices) has to be equal."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def pcpp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_23227_amd as m
    m.library()
    return m


def close(got, ref, magnitude, terms, what):
    """|got - ref| <= 8 (terms + 40) u magnitude, and half a unit of bf16 more for a bf16 result."""
    tol = 8 * (terms + 40) * U * magnitude + (2.0 ** -8 * (ref.abs() + 8 * (terms + 40) * U * magnitude) if got.dtype == BF16 else 0.0)
    got = got.double().cpu()
    assert got.shape == ref.shape, what
    off = (got - ref).abs() - tol
    worst = float(off.max()) if off.numel() else 0.0
    assert torch.isfinite(got).all() and worst <= 1e-40, (what, worst, float((got - ref).abs().max()))


# ---- activations in 8 bits ---------------------------------------------------------------------------------------

def packed_reference(x):
    """q, codes and values of rows, block by block, in binary64 (exact: powers of two)."""
    x = x.double().cpu().numpy()
    n, c = x.shape
    q, codes = np.zeros((n, c), np.int8), np.zeros((n, -(-c // 128) * 4), np.uint8)
    for b in range(-(-c // 32)):
        v = x[:, 32 * b:32 * b + 32]
        fine = np.isfinite(v).all(1)
        v = np.where(fine[:, None], v, 0.0)
        step = np.full(n, -126)                        # the smallest power of two with which nothing rounds past 127
        amax = np.abs(v).max(1)
        some = amax > 0
        step[some] = np.maximum(np.floor(np.log2(amax[some])).astype(int) - 8, -126)
        for _ in range(4):
            step = np.where(np.rint(np.ldexp(amax, -step)) > 127, step + 1, step)
        codes[:, b] = np.where(fine, step + 127, 255)
        q[:, 32 * b:32 * b + 32] = np.rint(np.ldexp(v, -step[:, None]))
    step = np.where(codes == 255, np.nan, np.ldexp(1.0, codes.astype(int) - 127))
    return q, codes, q * np.repeat(step, 32, axis=1)[:, :c]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (5, 8), (70, 20), (64, 32), (33, 33), (257, 64), (100, 91), (9, 129), (1000, 256), (17, 1000), (5, 1024)])
def test_pack_and_unpack(pcpp, n, c, dtype):
    g = torch.Generator().manual_seed(n * 1000 + c)
    x = torch.randn(n, c, generator=g) * torch.exp(4 * torch.randn(n, 1, generator=g))
    x[0, 0] = 127.5 * 2.0 ** -3                        # rounds past 127: takes the next power of two
    if n > 2:
        x[1] = 0.0
        x[2] *= 1e-39                                  # below the smallest power of two
    if n > 6:
        x[3, c // 2], x[4, 0], x[5, -1] = math.inf, math.nan, -math.inf
        x[6] = torch.arange(c) * 0.5                   # halves: to even
    x = x.to(dtype)
    p = pcpp.pcpp_act_pack(x.cuda())
    q, codes, values = packed_reference(x)
    assert np.array_equal(p.codes.cpu().numpy(), codes)
    assert np.array_equal(p.q.cpu().numpy(), q)
    for out in (F32, BF16):
        got = pcpp.pcpp_act_unpack(p, out)
        assert got.dtype == out and np.array_equal(got.double().cpu().numpy(), values, equal_nan=True)


def test_pack_of_no_rows(pcpp):
    p = pcpp.pcpp_act_pack(torch.empty(0, 40, device="cuda"))
    assert p.q.shape == (0, 40) and p.codes.shape == (0, 4) and pcpp.pcpp_act_unpack(p).shape == (0, 40)


@pytest.mark.parametrize("c_in,c_out,dtype,n,radius,t", [
    (32, 32, F32, 3000, 0.08, 3), (64, 128, BF16, 3000, 0.08, 3), (64, 64, BF16, 9000, 0.08, 3), (128, 64, BF16, 2500, 0.08, 2),
    (128, 128, BF16, 4000, 0.09, 3), (256, 256, BF16, 1500, 0.1, 3), (256, 256, F32, 400, 0.15, 2), (20, 36, F32, 2000, 0.08, 3),
    (20, 36, BF16, 2000, 0.08, 3), (91, 47, BF16, 1500, 0.09, 3), (91, 130, F32, 700, 0.1, 3), (1, 5, F32, 900, 0.1, 3),
    (3, 1, BF16, 900, 0.1, 3), (7, 40, BF16, 900, 0.1, 4), (8, 8, F32, 900, 0.1, 1), (200, 300, BF16, 600, 0.1, 3), (33, 1000, BF16, 200, 0.2, 2),
    (1000, 24, F32, 200, 0.2, 2),
])
def test_weight_gradient_from_packed_input(pcpp, c_in, c_out, dtype, n, radius, t):
    g = torch.Generator().manual_seed(c_in * 7 + c_out)
    xyz = torch.rand(n, 3, generator=g).cuda()
    T = pcpp.pcpp_build_triplets(xyz, xyz, radius, t)
    x = (torch.randn(n, c_in, generator=g) * torch.exp(torch.randn(c_in, generator=g))).to(dtype).cuda()
    x[::7] = 0.0
    dy = torch.randn(n, c_out, generator=g).to(dtype).cuda()
    p = pcpp.pcpp_act_pack(x)
    values = pcpp.pcpp_act_unpack(p, F32)
    got = pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, T)
    free = pcpp.Triplets(T.tri_o, T.tri_i, T.tri_k, T.seg_offsets, T.n_triplets, n, n, t, None, 0)
    assert torch.equal(got, pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, free))          # no plan needed; the same each time
    if dtype == BF16:                                                               # the values as bf16 rows: the same products
        assert torch.equal(got, pcpp.pcpp_mvmr_bwd_weight(values.to(BF16), dy, T))
    seg, o, i = T.seg_offsets.tolist(), T.tri_o.long().cpu(), T.tri_i.long().cpu()
    xd, dyd = values.double().cpu(), dy.double().cpu()
    longest = max(b - a for a, b in zip(seg[:-1], seg[1:]))
    for k in range(T.K):
        a, b = seg[k], seg[k + 1]
        ref = dyd[o[a:b]].T @ xd[i[a:b]]
        close(got[k], ref, dyd[o[a:b]].abs().T @ xd[i[a:b]].abs(), longest, ("dw", k))


@pytest.mark.parametrize("c_in,c_out,dtype", [
    (15, 4, F32), (16, 3, F32), (16, 9, F32), (17, 31, F32), (31, 32, F32), (32, 4, F32), (33, 17, F32), (5, 6, F32),
    (15, 24, BF16), (16, 8, BF16), (17, 31, BF16), (31, 64, BF16), (32, 128, BF16), (32, 3, BF16),
])
def test_weight_gradient_from_packed_rows_of_few_channels(pcpp, c_in, c_out, dtype):
    test_weight_gradient_from_packed_input(pcpp, c_in, c_out, dtype, 1500, 0.09, 3)


def test_weight_gradient_from_packed_input_without_triplets(pcpp):
    p = pcpp.pcpp_act_pack(torch.randn(10, 24, device="cuda"))
    dy = torch.randn(5, 16, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    T = pcpp.Triplets(none, none, none, torch.zeros(28, dtype=torch.int64, device="cuda"), 0, 10, 5, 3, None, 0)
    dw = torch.full((27, 16, 24), 3.0, device="cuda")
    assert not pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, T, dw=dw).any()


def test_non_finite_block_reaches_only_its_channels(pcpp):
    """A code of 255 is a NaN in the 32 channels of that row: the gradient is NaN in those columns of the row's cells and finite in the others'."""
    g = torch.Generator().manual_seed(1)
    n, c = 500, 96
    xyz = torch.rand(n, 3, generator=g).cuda()
    T = pcpp.pcpp_build_triplets(xyz, xyz, 0.1, 3)
    x = torch.randn(n, c, generator=g).cuda()
    x[17, 40] = math.inf
    got = pcpp.pcpp_mvmr_bwd_weight_packed(pcpp.pcpp_act_pack(x), torch.randn(n, 24, generator=g).cuda(), T)
    cells = T.tri_k[T.tri_i == 17].unique().long()
    assert torch.isnan(got[cells][:, :, 32:64]).all()
    assert torch.isfinite(got[:, :, :32]).all() and torch.isfinite(got[:, :, 64:]).all()


# ---- norms, gate, residual ---------------------------------------------------------------------------------------

def norm_reference(v, kind, eps, mag):
    """n(v), rstd, and the magnitude of what n(v) is formed from when v is off by its rounding at `mag`."""
    if kind == 0:
        return v, torch.ones(v.shape[0], 1, dtype=torch.float64), mag
    if kind == 2:
        mag = mag + mag.mean(1, keepdim=True)
        v = v - v.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + eps)
    n = v * rstd
    return n, rstd, rstd * mag + n.abs() * (rstd * mag * n.abs()).mean(1, keepdim=True)


def fwd_reference(x, f, gate, w_post, w_pre, post, pre, scale, eps):
    r, mag = x, x.abs()
    if f is not None:
        n, _, mn = norm_reference(f, post, eps, f.abs())
        sigma = torch.sigmoid(gate) if gate is not None else torch.ones(1, 1, dtype=torch.float64)
        r, mag = scale * x + sigma * (w_post * n), (scale * x).abs() + sigma * w_post.abs() * mn
        if gate is not None:                           # exp(-gate) in fp32: off by |gate| u
            mag = mag + sigma * w_post.abs() * n.abs() * gate.abs()
    if pre == 0:
        return r, None, mag, None
    n, _, mn = norm_reference(r, pre, eps, mag)
    return r, w_pre * n, mag, w_pre.abs() * mn


def norm_bwd_reference(y, ymag, n, nmag, rstd, kind):
    """gradient through n(v) of y, and its magnitude"""
    if kind == 0:
        return y, ymag
    d = y - n * (y * n).mean(1, keepdim=True)
    mag = ymag + nmag * (ymag * nmag).mean(1, keepdim=True)
    if kind == 2:
        d, mag = d - y.mean(1, keepdim=True), mag + ymag.mean(1, keepdim=True)
    return rstd * d, rstd * mag


CASES = [  # n, c, stream, dtype, post, pre, gate, scale
    (1, 256, BF16, BF16, 1, 1, "full", 1.0), (37, 32, F32, F32, 2, 2, "row", 0.5), (513, 64, F32, BF16, 1, 1, "full", 1.0),
    (300, 91, F32, BF16, 2, 2, "row", 0.75), (41, 20, F32, F32, 1, 2, "full", 1.0), (9, 1, F32, F32, 1, 1, "row", 1.0),
    (50, 3, BF16, BF16, 1, 1, "full", 1.0), (64, 7, F32, F32, 2, 1, "none", 1.0), (64, 8, F32, BF16, 1, 1, "row", 2.0),
    (33, 129, F32, F32, 2, 2, "full", 1.0), (40, 512, BF16, BF16, 1, 1, "full", 1.0), (21, 513, F32, BF16, 2, 2, "full", 1.0),
    (19, 1000, F32, F32, 1, 1, "row", 1.0), (12, 1024, BF16, BF16, 2, 2, "full", 1.0), (5000, 48, F32, F32, 1, 1, "full", 1.0),
    (70, 64, F32, F32, 0, 1, "full", 1.0), (70, 64, F32, BF16, 1, 0, "full", 1.0), (70, 40, F32, F32, 0, 0, "row", 1.0),
    (70, 96, F32, F32, 0, 2, "none", 0.5), (2100, 200, F32, BF16, 1, 1, "none", 1.0),
]


def block_inputs(n, c, stream, dtype, gate, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, c, generator=g) + 0.3).to(stream)
    f = (torch.randn(n, c, generator=g) * torch.exp(0.3 * torch.randn(c, generator=g)) - 0.2).to(dtype)
    ga = None if gate == "none" else torch.randn(n, c if gate == "full" else 1, generator=g).to(dtype)
    wp, wn = 1 + 0.3 * torch.randn(c, generator=g), 1 + 0.3 * torch.randn(c, generator=g)
    dr, dh = torch.randn(n, c, generator=g).to(stream), torch.randn(n, c, generator=g).to(dtype)
    return x, f, ga, wp, wn, dr, dh


def cuda(*ts):
    return [t.cuda() if t is not None else None for t in ts]


def wide(*ts):
    return [t.double().cpu() if t is not None else None for t in ts]


def half_way(c):
    """First row slot of a [n, 2 c + 1] tensor whose columns c + 1 .. hold a row: a slice, off any alignment."""
    return c + 1


@pytest.mark.parametrize("case", CASES, ids=lambda v: "-".join(str(e).replace("torch.", "") for e in v))
def test_block_norm_forward(pcpp, case):
    n, c, stream, dtype, post, pre, gate, scale = case
    x, f, ga, wp, wn, _, _ = block_inputs(n, c, stream, dtype, gate, 5)
    ref_r, ref_h, mag_r, mag_h = fwd_reference(*wide(x, f, ga, wp, wn), post, pre, scale, 1e-6)
    dx, df, dga, dwp, dwn = cuda(x, f, ga, wp, wn)
    both = torch.zeros(n, 2 * c + 1, dtype=dtype, device="cuda")
    both[:, half_way(c):] = df
    for fin in (df, both[:, half_way(c):]):                                         # contiguous, and columns of a wider tensor
        y = pcpp.pcpp_block_norm_fwd(dx, fin, dga, dwp, dwn, post_norm=post, pre_norm=pre, residual_scale=scale, pack_f=True, pack_h=pre > 0)
        close(y.r, ref_r, mag_r, c, "r")
        q, codes, _ = packed_reference(f)
        assert np.array_equal(y.f_packed.q.cpu().numpy(), q) and np.array_equal(y.f_packed.codes.cpu().numpy(), codes)
        if pre == 0:
            assert y.h is None
            continue
        close(y.h, ref_h, mag_h, c, "h")
        # the 8-bit copy: within a step's half of the unrounded h (a whole one where fp32 falls on the other side of a tie)
        values = pcpp.pcpp_act_unpack(y.h_packed, F32).double().cpu()
        step = torch.ldexp(torch.ones(1, dtype=torch.float64), y.h_packed.codes.cpu().double().repeat_interleave(32, 1)[:, :c] - 127)
        assert ((values - ref_h).abs() <= 0.5 * step + 8 * (c + 40) * U * mag_h).all()
    plain = pcpp.pcpp_block_norm_fwd(dx, df, dga, dwp, dwn, post_norm=post, pre_norm=pre, residual_scale=scale)
    assert torch.equal(plain.r, y.r) and (pre == 0 or torch.equal(plain.h, y.h)) and plain.f_packed is None and plain.h_packed is None


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda v: "-".join(str(e).replace("torch.", "") for e in v))
def test_block_norm_backward(pcpp, case, packed):
    n, c, stream, dtype, post, pre, gate, scale = case
    r, f, ga, wp, wn, dr, dh = block_inputs(n, c, stream, dtype, gate, 6)
    eps = 1e-6
    dev = cuda(dr, dh if pre else None, r if pre else None, f, ga, wp, wn)
    if packed:
        dev[3] = pcpp.pcpp_act_pack(dev[3])
        f = pcpp.pcpp_act_unpack(dev[3], F32)
    got = pcpp.pcpp_block_norm_bwd(*dev, post_norm=post, pre_norm=pre, residual_scale=scale, eps=eps, dtype=dtype)
    r, f, ga, wp, wn, dr, dh = wide(r, f, ga, wp, wn, dr, dh)
    d, dmag = dr, dr.abs()
    if pre:
        nr, rstd, mr = norm_reference(r, pre, eps, r.abs())
        y = wn * dh
        through, tmag = norm_bwd_reference(y, y.abs(), nr, mr, rstd, pre)
        d, dmag = d + through, dmag + tmag
        close(got.dw_pre, (dh * nr).sum(0), (dh.abs() * mr).sum(0), n + c, "dw_pre")
    else:
        assert got.dw_pre is None
    close(got.dx, scale * d, abs(scale) * dmag, c, "dx")
    sigma = torch.sigmoid(ga) if ga is not None else torch.ones(1, 1, dtype=torch.float64)
    off = 1 + ga.abs() if ga is not None else 1.0
    du, dumag = d * sigma, dmag * sigma * off
    nf, rstd, mf = norm_reference(f, post, eps, f.abs())
    df, mag = norm_bwd_reference(wp * du, wp.abs() * dumag, nf, mf, rstd, post)
    close(got.df, df, mag, c, "df")
    close(got.dw_post, (du * nf).sum(0), (dumag * mf).sum(0), n + c, "dw_post")      # (without a norm: of a scale for every channel)
    if ga is None:
        assert got.dgate is None
    else:
        # 1 - sigma is formed from sigma: off by u, not by a part of itself
        dg, gmag = du * (1 - sigma) * (wp * nf), dumag * wp.abs() * mf
        one = gate == "row"
        close(got.dgate, dg.sum(1, keepdim=True) if one else dg, gmag.sum(1, keepdim=True) if one else gmag, c, "dgate")
    again = pcpp.pcpp_block_norm_bwd(*dev, post_norm=post, pre_norm=pre, residual_scale=scale, eps=eps, dtype=dtype)
    for a, b in zip(vars(got).values(), vars(again).values()):
        assert a is None or torch.equal(a, b)                                       # sums in a fixed order


def test_block_norm_ends_of_a_network(pcpp):
    """In front of the first block there is only the norm; behind the last residual add nothing flows into r but through h."""
    n, c = 77, 40
    x, f, ga, wp, wn, dr, dh = cuda(*block_inputs(n, c, F32, F32, "full", 8))
    first = pcpp.pcpp_block_norm_fwd(x, w_pre=wn, pack_h=True)
    assert first.r is x
    ref = fwd_reference(x.double().cpu(), None, None, None, wn.double().cpu(), 0, 1, 1.0, 1e-6)
    close(first.h, ref[1], ref[3], c, "h")
    as_bf16 = pcpp.pcpp_block_norm_fwd(x, w_pre=wn, dtype=BF16).h
    close(as_bf16, ref[1], ref[3], c, "h bf16")
    whole = pcpp.pcpp_block_norm_bwd(dr, dh, x, None, None, None, wn)
    none = pcpp.pcpp_block_norm_bwd(None, dh, x, None, None, None, wn)
    assert whole.df is None and whole.dgate is None and whole.dw_post is None
    assert torch.equal(none.dw_pre, whole.dw_pre)
    assert torch.allclose(whole.dx - none.dx, dr, atol=1e-5)
    # neither a post norm nor a gate: what flows to f is what flows to r, and f itself is not needed
    got = pcpp.pcpp_block_norm_bwd(dr, dh, x, None, None, None, wn, post_norm=0, block=True)
    assert torch.equal(got.df, whole.dx)
    # no weights: ones
    y = pcpp.pcpp_block_norm_fwd(x, f, ga)
    o = torch.ones(c, device="cuda")
    z = pcpp.pcpp_block_norm_fwd(x, f, ga, o, o)
    assert torch.equal(y.r, z.r) and torch.equal(y.h, z.h)


def test_block_norm_of_no_rows_and_zero_rows(pcpp):
    c = 24
    e = torch.empty(0, c, device="cuda")
    y = pcpp.pcpp_block_norm_fwd(e, e)
    assert y.r.shape == (0, c) and y.h.shape == (0, c)
    g = pcpp.pcpp_block_norm_bwd(e, e, e, e)
    assert not g.dw_post.any() and not g.dw_pre.any()
    z = torch.zeros(3, c, device="cuda")
    for kind in (1, 2):
        y = pcpp.pcpp_block_norm_fwd(z, z, post_norm=kind, pre_norm=kind)
        assert not y.r.any() and not y.h.any()


def test_block_norm_keeps_non_finite_rows_apart(pcpp):
    x, f, ga, wp, wn, dr, dh = cuda(*block_inputs(40, 72, F32, F32, "full", 9))
    ref, back = pcpp.pcpp_block_norm_fwd(x, f, ga, wp, wn), pcpp.pcpp_block_norm_bwd(dr, dh, x, f, ga, wp, wn)
    f2 = f.clone()
    f2[7, 3], f2[20, 70] = math.nan, math.inf
    y, b = pcpp.pcpp_block_norm_fwd(x, f2, ga, wp, wn), pcpp.pcpp_block_norm_bwd(dr, dh, x, f2, ga, wp, wn)
    rows = torch.ones(40, dtype=torch.bool, device="cuda")
    rows[7] = rows[20] = False
    assert torch.isnan(y.h[~rows]).all() and torch.equal(y.h[rows], ref.h[rows]) and torch.equal(y.r[rows], ref.r[rows])
    assert torch.equal(b.df[rows], back.df[rows]) and torch.equal(b.dx, back.dx)
    # a gate's NaN, and gates so large that they are 0 and 1
    ga2 = ga.clone()
    ga2[3, 5], ga2[8, 1], ga2[9, 1], ga2[10, 1], ga2[11, 1] = math.nan, math.inf, -math.inf, 1e30, -1e30
    y, b = pcpp.pcpp_block_norm_fwd(x, f, ga2, wp, wn), pcpp.pcpp_block_norm_bwd(dr, dh, x, f, ga2, wp, wn)
    assert torch.isnan(y.r[3, 5]) and torch.isnan(y.h[3]).all() and torch.isnan(b.df[3]).all() and torch.isnan(b.dgate[3, 5])
    assert torch.equal(y.r[9, 1], x[9, 1]) and torch.equal(y.r[11, 1], x[11, 1])
    assert not b.dgate[8:12, 1].any() and torch.isfinite(b.df[4:20]).all()
    one = pcpp.pcpp_block_norm_bwd(dr, dh, x, f, ga[:, :1].clone().fill_(math.nan), wp, wn)
    assert torch.isnan(one.df).all() and torch.isnan(one.dgate).all() and torch.equal(one.dx, back.dx)


@pytest.mark.parametrize("kind,gate", [(1, "full"), (2, "row"), (1, "none")])
def test_block_norm_gradient_against_differences(pcpp, kind, gate):
    """L = <dr, r> + <dh, h> in one direction: central differences at e = 2^-7 are off by e^2 / 6 times a third derivative and by the rounding
    of 2 n c fp32 values over e; 2e-3 of the products' norm covers both."""
    n, c = 64, 40
    x, f, ga, wp, wn, dr, dh = cuda(*block_inputs(n, c, F32, F32, gate, 10))
    how = dict(post_norm=kind, pre_norm=kind, residual_scale=0.8)
    fwd = lambda *a: pcpp.pcpp_block_norm_fwd(*a, **how)  # noqa: E731
    loss = lambda y: float((dr.double() * y.r.double()).sum() + (dh.double() * y.h.double()).sum())  # noqa: E731
    y = fwd(x, f, ga, wp, wn)
    grads = pcpp.pcpp_block_norm_bwd(dr, dh, y.r, f, ga, wp, wn, **how)
    ins = {"x": x, "f": f, "gate": ga, "w_post": wp, "w_pre": wn}
    of = {"x": grads.dx, "f": grads.df, "gate": grads.dgate, "w_post": grads.dw_post, "w_pre": grads.dw_pre}
    g = torch.Generator(device="cuda").manual_seed(3)
    for name, v in ins.items():
        if v is None:
            continue
        way = torch.randn(v.shape, generator=g, device="cuda")
        e = 2.0 ** -7
        plus, minus = ({**ins, name: v + s * e * way} for s in (1, -1))
        slope = (loss(fwd(*plus.values())) - loss(fwd(*minus.values()))) / (2 * e)
        want = float((of[name].double() * way.double()).sum())
        scale = float(of[name].double().norm() * way.double().norm())
        assert abs(slope - want) <= 2e-3 * scale, (name, slope, want, scale)


def test_block_norm_without_eps(pcpp):
    """eps = 0: rows that a wave holds past the last one have no norm, and must not reach the weights' gradients."""
    for n, c in ((37, 32), (5, 91), (1, 7)):
        r, f, ga, wp, wn, dr, dh = block_inputs(n, c, F32, F32, "full", 11)
        got = pcpp.pcpp_block_norm_bwd(*cuda(dr, dh, r, f, ga, wp, wn), eps=0.0)
        r, dh = wide(r, dh)
        nr, _, mr = norm_reference(r, 1, 0.0, r.abs())
        close(got.dw_pre, (dh * nr).sum(0), (dh.abs() * mr).sum(0), n + c, "dw_pre")
        assert torch.isfinite(got.dw_post).all() and torch.isfinite(got.df).all()


# ---- log probabilities -------------------------------------------------------------------------------------------

def head_reference(x, labels, n_top):
    x = x.double().cpu()
    n, v = x.shape
    m = x.amax(1, keepdim=True)
    some = m > -math.inf
    z = torch.exp(x - torch.where(some, m, 0.0))
    total = z.sum(1, keepdim=True)
    lse = m + torch.log(total)
    lp = torch.where(some, (x - torch.where(some, m, 0.0)) - torch.log(total), -math.inf)
    p = torch.where(some, z / total, 0.0)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    labels = labels.long().cpu()
    given = (labels >= 0) & (labels < v)
    picked = lp.gather(1, labels.clamp(0, v - 1)[:, None])[:, 0]
    order = torch.sort(-x, dim=1, stable=True).indices[:, :n_top]                  # (-0 and 0 are equal)
    return lse[:, 0], torch.where(given, picked, 0.0), entropy, lp.gather(1, order), order, p, lp, given


def head_terms(v):
    """Terms that a 32-bit sum of a row goes through one after the other at most: a lane's share, then the lanes and blocks."""
    return v / 64 + 64


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,v,n_top,mask", [
    (1, 1, 1, 0.0), (5, 2, 2, 0.0), (1000, 17, 3, 0.0), (77, 32, 32, 0.5), (64, 33, 20, 0.0), (31, 64, 0, 0.0), (20, 100, 64, 0.7), (65, 256, 5, 0.0),
    (9, 257, 1, 0.0), (40, 512, 20, 0.9), (7, 513, 20, 0.9), (3, 1000, 64, 0.0), (300, 1031, 5, 0.0), (2, 4097, 8, 0.3), (1, 9999, 20, 0.0),
    (1, 131072, 20, 0.3), (3, 70001, 64, 0.0), (1100, 2050, 1, 0.0),
])
def test_log_probs(pcpp, n, v, n_top, mask, dtype):
    g = torch.Generator().manual_seed(n + v)
    x = (3 * torch.randn(n, v, generator=g) + 5 * torch.randn(n, 1, generator=g)).to(dtype)
    x = torch.where(torch.rand(n, v, generator=g) < mask / 2, -math.inf, x)
    x = torch.where(torch.rand(n, v, generator=g) < mask / 2, torch.finfo(dtype).min, x)
    if n > 4:
        x[1] = -math.inf                               # no class at all
        x[2] = torch.finfo(dtype).min                  # all at the type's lowest value: all equally probable
        x[3] = 0.0
        x[3, ::2] = -0.0                               # equal: the lowest indices first
        x[4] = -math.inf
        x[4, v // 2] = 1.0                             # a single class
    labels = torch.randint(v, (n,), generator=g, dtype=torch.int32)
    labels[::5] = torch.tensor([-1, v, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)[torch.arange(len(labels[::5])) % 4]
    lse, log_prob, entropy, top, index, p, lp, given = head_reference(x, labels, n_top)
    some = torch.isfinite(lse)
    wide_ = torch.full((n, v + 3), 7.0, dtype=dtype, device="cuda")
    wide_[:, 1:v + 1] = x.cuda()
    terms = head_terms(v)
    dl, dh = torch.randn(n, generator=g), torch.randn(n, generator=g)
    dl_ref = torch.where(given & some, dl.double(), 0.0)[:, None]
    hit = torch.zeros(n, v, dtype=torch.float64)
    hit[torch.arange(n), labels.long().clamp(0, v - 1)] = 1.0
    flat = torch.where(p > 0, p * (lp + entropy[:, None]), 0.0)
    d_ref = torch.where(some[:, None], dl_ref * (hit - p) - dh.double()[:, None] * flat, 0.0)
    # p is off by the rounding of its logarithm
    size = 1 + torch.where(p > 0, lp.abs(), 0.0)
    d_mag = torch.where(some[:, None], (dl_ref.abs() * (hit + p) + dh.double().abs()[:, None] * torch.where(p > 0, p * (lp.abs() + entropy[:, None] + 1), 0.0)) * size, 0.0)
    for logits in (x.cuda(), wide_[:, 1:v + 1]):                                    # contiguous, and a slice off any alignment
        y = pcpp.pcpp_log_probs_fwd(logits, labels.cuda(), n_top)
        assert torch.equal(y.top_index.cpu().long(), index)
        for got, ref, what in ((y.lse, lse, "lse"), (y.log_prob, log_prob, "log_prob"), (y.top_log_prob, top, "top")):
            got, fine = got.double().cpu(), torch.isfinite(ref)
            assert torch.equal(torch.isfinite(got), fine) and torch.equal(got[~fine], ref[~fine]), what
            close(got[fine].float(), ref[fine], 1 + ref[fine].abs(), terms, what)
        close(y.entropy, entropy, 1 + entropy + torch.where(p > 0, p * lp.abs(), 0.0).sum(1), terms, "entropy")
        got = pcpp.pcpp_log_probs_bwd(logits, labels.cuda(), y, dl.cuda(), dh.cuda())
        close(got, d_ref, d_mag, terms, "d_logits")
        other = pcpp.pcpp_log_probs_bwd(logits, labels.cuda(), y, dl.cuda())
        close(other, torch.where(some[:, None], dl_ref * (hit - p), 0.0), dl_ref.abs() * (hit + p) * size, terms, "d_logits, no entropy")
        place = logits.clone() if logits.is_contiguous() else logits
        assert torch.equal(pcpp.pcpp_log_probs_bwd(place, labels.cuda(), y, dl.cuda(), dh.cuda(), out=place), got)   # in place
    assert (wide_[:, 0] == 7).all() and (wide_[:, v + 1:] == 7).all()               # the columns beside the slice are as they were


def test_log_probs_without_labels_or_rows(pcpp):
    x = torch.randn(6, 40, device="cuda")
    y = pcpp.pcpp_log_probs_fwd(x, None, 4)
    assert y.log_prob is None
    z = pcpp.pcpp_log_probs_fwd(x, torch.zeros(6, dtype=torch.int32, device="cuda"), 4)
    assert torch.equal(y.entropy, z.entropy) and torch.equal(y.top_index, z.top_index)
    e = pcpp.pcpp_log_probs_fwd(torch.empty(0, 40, device="cuda"), None, 4)
    assert e.top_index.shape == (0, 4)


@pytest.mark.parametrize("v", [40, 700, 9000])
def test_log_probs_of_rows_that_are_not_finite(pcpp, v):
    """NaN and +inf reach everything of their row but its indices, and no other row."""
    x = torch.randn(6, v, generator=torch.Generator().manual_seed(v))
    fine = pcpp.pcpp_log_probs_fwd(x.cuda(), torch.zeros(6, dtype=torch.int32).cuda(), 5)
    x[1, v // 3], x[4, v - 1] = math.nan, math.inf
    labels = torch.zeros(6, dtype=torch.int32).cuda()
    y = pcpp.pcpp_log_probs_fwd(x.cuda(), labels, 5)
    d = pcpp.pcpp_log_probs_bwd(x.cuda(), labels, y, torch.ones(6).cuda(), torch.ones(6).cuda())
    bad = torch.tensor([False, True, False, False, True, False])
    for t, u in ((y.lse, fine.lse), (y.log_prob, fine.log_prob), (y.entropy, fine.entropy), (y.top_log_prob, fine.top_log_prob)):
        assert torch.isnan(t.cpu()[bad]).all() and torch.equal(t.cpu()[~bad], u.cpu()[~bad])
    assert torch.isnan(d.cpu()[bad]).all() and torch.isfinite(d.cpu()[~bad]).all()
    order = torch.sort(-torch.where(torch.isnan(x), -math.inf, x), dim=1, stable=True).indices[:, :5]
    assert torch.equal(y.top_index.cpu().long(), order)                             # a NaN ranks as -inf


@pytest.mark.parametrize("order", ["ascending", "descending", "equal"])
def test_alternatives_of_sorted_rows(pcpp, order):
    """Every element of an ascending row passes the list so far; of equal ones the first are kept."""
    v = 20_000
    x = torch.arange(v, dtype=F32)[None] / v
    x = {"ascending": x, "descending": -x, "equal": 0 * x}[order]
    for n in (1, 2):
        y = pcpp.pcpp_log_probs_fwd(x.repeat(n, 1).cuda(), None, 64)
        want = torch.arange(v - 1, v - 65, -1) if order == "ascending" else torch.arange(64)
        assert torch.equal(y.top_index.cpu().long(), want.repeat(n, 1))


def test_log_probs_gradient_against_differences(pcpp):
    """L = <dl, log_prob> + <dh, entropy>: central differences at e = 2^-6, off by e^2 / 6 times a third derivative and rounding over e."""
    n, v = 50, 60
    g = torch.Generator(device="cuda").manual_seed(4)
    x, way = torch.randn(n, v, generator=g, device="cuda"), torch.randn(n, v, generator=g, device="cuda")
    labels = torch.randint(v, (n,), generator=g, device="cuda", dtype=torch.int32)
    dl, dh = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")

    def loss(x):
        y = pcpp.pcpp_log_probs_fwd(x, labels)
        return float((dl.double() * y.log_prob.double()).sum() + (dh.double() * y.entropy.double()).sum())

    d = pcpp.pcpp_log_probs_bwd(x, labels, pcpp.pcpp_log_probs_fwd(x, labels), dl, dh)
    e = 2.0 ** -6
    slope = (loss(x + e * way) - loss(x - e * way)) / (2 * e)
    want = float((d.double() * way.double()).sum())
    assert abs(slope - want) <= 2e-3 * float(d.double().norm() * way.double().norm())


# ---- streams, graphs, large tensors ------------------------------------------------------------------------------

def everything(pcpp, s):
    y = pcpp.pcpp_block_norm_fwd(s["x"], s["f"], s["gate"], s["wp"], s["wn"], pack_f=True, pack_h=True)
    b = pcpp.pcpp_block_norm_bwd(s["dr"], s["dh"], y.r, y.f_packed, s["gate"], s["wp"], s["wn"])
    dw = pcpp.pcpp_mvmr_bwd_weight_packed(y.h_packed, s["dy"], s["T"])
    lp = pcpp.pcpp_log_probs_fwd(s["logits"], s["labels"], 5)
    d = pcpp.pcpp_log_probs_bwd(s["logits"], s["labels"], lp, s["dl"], s["dl"])
    return [y.r, y.h, b.dx, b.df, b.dgate, b.dw_post, b.dw_pre, dw, lp.log_prob, lp.entropy, lp.top_log_prob, lp.top_index, d]


def everything_inputs(pcpp, seed, n=1500, c=72):
    x, f, ga, wp, wn, dr, dh = cuda(*block_inputs(n, c, F32, BF16, "full", seed))
    g = torch.Generator(device="cuda").manual_seed(seed)
    xyz = torch.rand(n, 3, generator=g, device="cuda")
    return dict(x=x, f=f, gate=ga, wp=wp, wn=wn, dr=dr, dh=dh, T=pcpp.pcpp_build_triplets(xyz, xyz, 0.1, 3),
                dy=torch.randn(n, 40, generator=g, device="cuda").to(BF16), logits=torch.randn(4, 30_001, generator=g, device="cuda").to(BF16),
                labels=torch.arange(4, dtype=torch.int32, device="cuda"), dl=torch.randn(4, generator=g, device="cuda"))


def test_other_streams(pcpp):
    s = everything_inputs(pcpp, 1)
    ref = everything(pcpp, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = everything(pcpp, s)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_captured_in_a_graph(pcpp):
    """The whole set in one graph, replayed with other inputs and eager work between: every replay as the eager calls."""
    s, other = everything_inputs(pcpp, 2), everything_inputs(pcpp, 3)
    everything(pcpp, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        everything(pcpp, s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything(pcpp, s)
    for k in range(4):
        for name in ("x", "f", "gate", "dr", "dh", "dy", "logits", "dl"):
            s[name].copy_(other[name] * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        ref = everything(pcpp, s)
        assert all(torch.equal(a, b) for a, b in zip(ref, out)), k


def test_rows_past_32_bits(pcpp):
    """Tensors of more than 2^31 elements and 4 GiB: the last rows as in a call of their own."""
    if torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("needs 64 GiB")
    n, c, tail = 2_200_000, 1024, 1000
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n, c, generator=g, device="cuda", dtype=BF16)
    p = pcpp.pcpp_act_pack(x)
    q = pcpp.pcpp_act_pack(x[-tail:].contiguous())
    assert torch.equal(p.q[-tail:], q.q) and torch.equal(p.codes[-tail:], q.codes)
    assert torch.equal(pcpp.pcpp_act_unpack(p)[-tail:], pcpp.pcpp_act_unpack(q))
    y, z = pcpp.pcpp_block_norm_fwd(x, x, x), pcpp.pcpp_block_norm_fwd(*[x[-tail:].contiguous()] * 3)
    assert torch.equal(y.r[-tail:], z.r) and torch.equal(y.h[-tail:], z.h)
    del y
    y, z = pcpp.pcpp_block_norm_bwd(x, x, x, p, x), pcpp.pcpp_block_norm_bwd(*[x[-tail:].contiguous()] * 3, q, x[-tail:].contiguous())
    assert torch.equal(y.dx[-tail:], z.dx) and torch.equal(y.df[-tail:], z.df) and torch.equal(y.dgate[-tail:], z.dgate)
    del y, p
    for rows, v in ((n * c // 131_072, 131_072), (n * c // 500, 500)):
        logits = x.view(-1)[:rows * v].view(rows, v)
        labels = torch.randint(v, (rows,), generator=g, device="cuda", dtype=torch.int32)
        ones = torch.ones(rows, device="cuda")
        y = pcpp.pcpp_log_probs_fwd(logits, labels, 3)
        z = pcpp.pcpp_log_probs_fwd(logits[-2000:].contiguous(), labels[-2000:].contiguous(), 3)
        assert torch.equal(y.log_prob[-2000:], z.log_prob) and torch.equal(y.top_index[-2000:], z.top_index)
        d = pcpp.pcpp_log_probs_bwd(logits, labels, y, ones, ones)[-2000:]
        assert torch.equal(d, pcpp.pcpp_log_probs_bwd(logits[-2000:], labels[-2000:].contiguous(), z, ones[-2000:].contiguous(), ones[-2000:].contiguous()))


def test_packed_weight_gradient_past_32_bits(pcpp):
    """A bf16 copy of x of more than 4 GiB: the kernel that needs the plan, and a refusal without one."""
    if torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("needs 64 GiB")
    n_in, n_out, c_in, c_out = 2_200_000, 70, 1024, 8
    g = torch.Generator(device="cuda").manual_seed(6)
    xyz = torch.rand(n_in, 3, generator=g, device="cuda")
    centres = xyz[-n_out:].contiguous()
    T = pcpp.pcpp_build_triplets(xyz, centres, 0.01, 2)
    p = pcpp.pcpp_act_pack(torch.randn(n_in, c_in, generator=g, device="cuda", dtype=BF16))
    dy = torch.randn(n_out, c_out, generator=g, device="cuda").to(BF16)
    got = pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, T)
    o, i, k = (t.long() for t in (T.tri_o, T.tri_i, T.tri_k))
    x, d = pcpp.pcpp_act_unpack(pcpp.Packed(p.q[i].contiguous(), p.codes[i].contiguous()), F32).double().cpu(), dy[o].double().cpu()
    for cell in range(T.K):
        at = (k == cell).cpu()
        close(got[cell], d[at].T @ x[at], d[at].abs().T @ x[at].abs(), int(at.sum()), ("dw", cell))
    free = pcpp.Triplets(T.tri_o, T.tri_i, T.tri_k, T.seg_offsets, T.n_triplets, n_in, n_out, 2, None, 0)
    with pytest.raises(pcpp.PcppError) as e:
        pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, free)
    assert e.value.code == -1 and "plan" in str(e.value)


def test_refusals_of_tensors(pcpp):
    """What does not fit is refused before the library is called."""
    x, f = torch.randn(6, 40, device="cuda"), torch.randn(6, 40, device="cuda")
    p = pcpp.pcpp_act_pack(x)
    i32 = torch.zeros(6, dtype=torch.int32, device="cuda")
    y = pcpp.pcpp_log_probs_fwd(x, i32)
    for call in (lambda: pcpp.pcpp_act_pack(x.cpu()), lambda: pcpp.pcpp_act_pack(x.t()), lambda: pcpp.pcpp_act_pack(x[0]),
                 lambda: pcpp.pcpp_act_unpack(pcpp.Packed(p.q, p.codes[:5])), lambda: pcpp.pcpp_act_unpack(pcpp.Packed(p.codes, p.q)),
                 lambda: pcpp.pcpp_act_unpack(p, out=torch.empty(6, 41, device="cuda")), lambda: pcpp.pcpp_block_norm_fwd(x, f[:5]),
                 lambda: pcpp.pcpp_block_norm_fwd(x, f, f[:, :2]), lambda: pcpp.pcpp_block_norm_fwd(x, f, f.to(BF16)), lambda: pcpp.pcpp_block_norm_fwd(x, f.t()),
                 lambda: pcpp.pcpp_block_norm_fwd(x, f, None, x[0, :39]), lambda: pcpp.pcpp_block_norm_fwd(x, f, None, x[0].to(BF16)),
                 lambda: pcpp.pcpp_block_norm_bwd(None, None, x, f), lambda: pcpp.pcpp_block_norm_bwd(x, x, x.to(BF16), f),
                 lambda: pcpp.pcpp_block_norm_bwd(x[:5], x, x, f), lambda: pcpp.pcpp_block_norm_bwd(x.t(), x, x, f),
                 lambda: pcpp.pcpp_log_probs_fwd(x, i32.long()), lambda: pcpp.pcpp_log_probs_fwd(x, i32[:5]), lambda: pcpp.pcpp_log_probs_fwd(x.t()),
                 lambda: pcpp.pcpp_log_probs_fwd(x[0]), lambda: pcpp.pcpp_log_probs_bwd(x[:5], None, y),
                 lambda: pcpp.pcpp_log_probs_bwd(x, i32, y, x[:, 0]), lambda: pcpp.pcpp_log_probs_bwd(x, i32, y, out=x[:, :39])):
        with pytest.raises((AssertionError, TypeError)):
            call()
    for call in (lambda: pcpp.pcpp_act_pack(x.half()), lambda: pcpp.pcpp_act_unpack(p, torch.float16), lambda: pcpp.pcpp_block_norm_fwd(x.half(), f.half()),
                 lambda: pcpp.pcpp_log_probs_fwd(x.double()), lambda: pcpp.pcpp_block_norm_fwd(None, f), lambda: pcpp.pcpp_log_probs_fwd("x")):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: pcpp.pcpp_block_norm_fwd(x, f, pre_norm=7), lambda: pcpp.pcpp_block_norm_fwd(x, f, eps=-1.0),
                 lambda: pcpp.pcpp_log_probs_fwd(x, None, 41), lambda: pcpp.pcpp_act_pack(torch.randn(2, 1025, device="cuda")),
                 lambda: pcpp.pcpp_block_norm_bwd(x, x, x, None, f)):
        with pytest.raises(pcpp.PcppError):
            call()
