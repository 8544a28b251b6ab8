"""The operators around the convolution held to what 32 bits give, where a sum over a whole row, cell or cloud would hide a lost part of it.

u = 2^-24 is the rounding of fp32.  Every bound counts the roundings that a result goes through, and every test says, from the oracle alone, which
mistake would pass it."""
import math

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


# ---- weight gradient from 8 bits beside an fp32 dy: all of dy's 24 bits take part -----------------------------------------------------

def cloud(pcpp, n, radius, t, seed):
    xyz = torch.rand(n, 3, generator=torch.Generator().manual_seed(seed)).cuda()
    return pcpp.pcpp_build_triplets(xyz, xyz, radius, t)


def weight_reference(x, dy, T):
    """dW in binary64"""
    seg, o, i = T.seg_offsets.tolist(), T.tri_o.long().cpu(), T.tri_i.long().cpu()
    x, dy = x.double().cpu(), dy.double().cpu()
    return torch.stack([dy[o[a:b]].T @ x[i[a:b]] for a, b in zip(seg[:-1], seg[1:])])


WEIGHT_SHAPES = [(32, 32), (64, 64), (20, 36), (91, 130), (1, 5), (8, 8), (5, 6), (33, 17), (256, 256), (16, 9), (1000, 24), (3, 1)]


@pytest.mark.parametrize("c_in,c_out", WEIGHT_SHAPES)
def test_packed_weight_gradient_of_exact_sums(pcpp, c_in, c_out):
    """x is 0 or 1 and dy = 1 + a 2^-9 + b 2^-18, three bf16 numbers one below the other.  Sums of a cell stay under 64, so they are whole multiples of
    2^-18 in 24 bits: nothing is rounded on any way through, and the result has to be equal."""
    n = 2500 if c_in * c_out < 20_000 else 900
    T = cloud(pcpp, n, 0.13 if n == 2500 else 0.2, 3, c_in + c_out)
    g = torch.Generator().manual_seed(c_in * 31 + c_out)
    longest = int((T.seg_offsets[1:] - T.seg_offsets[:-1]).max())
    x = (torch.rand(n, c_in, generator=g) < 20.0 / longest).float()
    a, b = ((torch.rand(n, c_out, generator=g) < 0.9).float() for _ in range(2))
    dy = 1 + a * 2.0 ** -9 + b * 2.0 ** -18
    ref = weight_reference(x, dy, T)
    assert float(ref.max()) < 64 and longest > 64
    for short in (1 + 0 * a, 1 + a * 2.0 ** -9):       # dy's first term alone, its first two
        assert not torch.equal(weight_reference(x, short, T), ref)
    p = pcpp.pcpp_act_pack(x.cuda())
    assert torch.equal(pcpp.pcpp_act_unpack(p, F32).cpu(), x)
    assert torch.equal(pcpp.pcpp_mvmr_bwd_weight_packed(p, dy.cuda(), T).double().cpu(), ref)


@pytest.mark.parametrize("c_in,c_out", WEIGHT_SHAPES)
def test_packed_weight_gradient_in_fp32_keeps_24_bits(pcpp, c_in, c_out):
    """Random rows: dy's three terms leave 2^-24 of it, and a wave adds a few tens of windows of 32 triplets, the waves and chunks as many sums: as
    independent roundings 2^-24 times the root of under 100, 6e-7 of the norm.  Without dy's third term it would be 2^-18 and more, 4e-6."""
    n = 2500 if c_in * c_out < 20_000 else 900
    T = cloud(pcpp, n, 0.13 if n == 2500 else 0.2, 3, c_in + c_out)
    g = torch.Generator().manual_seed(c_in * 31 + c_out)
    p = pcpp.pcpp_act_pack(torch.randn(n, c_in, generator=g).cuda())
    x, dy = pcpp.pcpp_act_unpack(p, F32), torch.randn(n, c_out, generator=g)
    first = dy.bfloat16().float()
    two = first + (dy - first).bfloat16().float()
    ref, short = weight_reference(x, dy, T), weight_reference(x, two, T)
    assert float((short - ref).norm() / ref.norm()) > 1e-6
    got = pcpp.pcpp_mvmr_bwd_weight_packed(p, dy.cuda(), T).double().cpu()
    assert float((got - ref).norm() / ref.norm()) <= 1e-6


# ---- log probabilities: every class of a row counts ---------------------------------------------------------------------------------

def head_reference(x, labels):
    """log S, T / S and what the bounds need, in binary64."""
    x = x.double().cpu()
    m = x.amax(1, keepdim=True)
    d = x - m
    z = torch.exp(d)
    s = z.sum(1, keepdim=True)
    p, log_s = z / s, torch.log(s)
    at = labels.long().cpu()[:, None]
    lp = d - log_s
    return m[:, 0], log_s[:, 0], lp, p, lp.gather(1, at)[:, 0], -(p * lp).sum(1), (p * d * d).sum(1)


# lengths about a step of a lane's eight classes, of a wave's and a block's, and a split's 4096, with rests of one class to one short
LENGTHS = [513, 519, 1023, 1025, 1031, 2047, 2056, 4095, 4097, 4103, 8191, 8193, 8200, 9999, 12_295, 16_385, 65_537, 70_001, 131_071, 131_072]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [9, 17, 63, 65, 255, 257, 511] + LENGTHS)
def test_log_probs_of_equal_classes(pcpp, v, dtype):
    """v equal logits: S is v exactly (sums of ones under 2^24), so log S is off by the logarithm alone, two roundings of a number under 17 and one of its product
    with log 2: under 4 u log v.  A class lost or counted twice changes it by 1 / v, which is more."""
    bound = 4 * U * math.log(v)
    assert 1 / (v + 1) > 1.3 * bound
    for n in (1, 3, 300, 1100) if v < 20_000 else (1, 3, 70):
        x = torch.full((n, v), 1.5, dtype=dtype, device="cuda")
        labels = torch.arange(n, dtype=torch.int32, device="cuda") % v
        for n_top in (0, 3):
            y = pcpp.pcpp_log_probs_fwd(x, labels, n_top)
            m, log_s = y.max_log_sum.double().unbind(1)
            assert (m == 1.5).all() and float((log_s - math.log(v)).abs().max()) <= bound, (n, n_top)
            assert float((y.log_prob.double() + math.log(v)).abs().max()) <= bound
            assert float((y.entropy.double() - math.log(v)).abs().max()) <= bound
            if n_top:
                assert torch.equal(y.top_index, torch.arange(3, dtype=torch.int32, device="cuda").repeat(n, 1))
        d = pcpp.pcpp_log_probs_bwd(x, labels, y, torch.ones(n, device="cuda")).double()
        hit = torch.arange(v, device="cuda") == labels[:, None]
        size = 2.0 ** -8 if dtype == BF16 else 0.0
        # p is off by its logarithm's error, the exponent's rounding (log v times 2 u) and its own
        off = (d - (hit.double() - 1 / v)).abs() - (hit.double() + 1 / v) * size
        assert float((off - (1 / v) * (bound + (2 * math.log(v) + 4) * U) - hit.double() * 2 * U).max()) <= 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", LENGTHS)
def test_log_probs_to_32_bits(pcpp, v, dtype):
    """Random rows.  exp(d) is off by (1.5 |d| + 2) u of itself; S by that over all classes, at most 1.5 E|d| + 2 <= 1.5 sqrt(E d^2) + 2, and by
    a tree of additions, under 8 u as independent roundings; log S by three more.  T / S by the same times |d|: (1.5 E d^2 + 10 E|d|) u.  With
    E d^2 <= 60 here that is under 2e-6 (1 + |log S|) and 2e-6 (1 + log S + E d^2); a log probability has its two subtractions, of x and m, beside."""
    for n in (1, 3, 1100 if v < 5000 else 40 if v < 20_000 else 9):
        g = torch.Generator().manual_seed(v + n)
        x = (2 * torch.randn(n, v, generator=g) + torch.randn(n, 1, generator=g)).to(dtype)
        labels = torch.randint(v, (n,), generator=g, dtype=torch.int32)
        labels[0] = v - 1                              # the last class of a rest
        m, log_s, lp, p, picked, entropy, spread = head_reference(x, labels)
        assert float(spread.max()) <= 60
        y = pcpp.pcpp_log_probs_fwd(x.cuda(), labels.cuda(), 4)
        gm, glog = y.max_log_sum.double().cpu().unbind(1)
        assert torch.equal(gm, m) and ((glog - log_s).abs() <= 2e-6 * (1 + log_s)).all()
        assert ((y.log_prob.double().cpu() - picked).abs() <= 2e-6 * (1 + picked.abs() + log_s)).all()
        top, index = torch.sort(-x.double(), dim=1, stable=True)
        assert torch.equal(y.top_index.cpu().long(), index[:, :4])
        assert ((y.top_log_prob.double().cpu() - lp.gather(1, index[:, :4])).abs() <= 2e-6 * (1 + log_s[:, None] + m[:, None].abs())).all()
        assert ((y.entropy.double().cpu() - entropy).abs() <= 2e-6 * (1 + log_s + spread)).all()
        dl, dh = torch.randn(n, generator=g), torch.randn(n, generator=g)
        got = pcpp.pcpp_log_probs_bwd(x.cuda(), labels.cuda(), y, dl.cuda(), dh.cuda()).double().cpu()
        hit = torch.nn.functional.one_hot(labels.long(), v).double()
        dl, dh = dl.double()[:, None], dh.double()[:, None]
        ref = dl * (hit - p) - dh * p * (lp + entropy[:, None])
        parts = dl.abs() * (hit + p) + dh.abs() * p * (lp.abs() + entropy[:, None] + 1)
        # p is off by what its logarithm is: the row's log S, and the roundings of a number of its size
        tol = parts * (2e-6 * (1 + log_s + spread)[:, None] + 4 * U * lp.abs())
        if dtype == BF16:
            tol = tol + 2.0 ** -8 * (ref.abs() + tol)
        assert ((got - ref).abs() <= tol + 1e-40).all()


# ---- gradients of the norms' weights: every row of a large cloud counts ----------------------------------------------------------------

@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n,c,stream,dtype,kind,gate", [
    (70_001, 64, F32, BF16, 1, "full"), (70_001, 64, F32, F32, 2, "row"), (9001, 520, F32, F32, 1, "full"), (9001, 520, BF16, BF16, 2, "none"),
    (200_003, 32, F32, F32, 1, "row"), (70_003, 91, F32, BF16, 2, "full"), (140_001, 7, F32, F32, 1, "full"),
])
def test_weights_gradients_over_many_rounds(pcpp, n, c, stream, dtype, kind, gate, packed):
    """More rows than the largest launch holds at a time, so that every block goes round and all its sums join.  A column's sum goes through the rounds of
    a lane (under 8), log2 of the lanes (4), the waves (4) and the blocks' sums (1024 / 64 + 2 + 16), 50 additions at most, and a term, formed from
    statistics of a row in registers (8 to 16 elements and 6 steps over the lanes, each norm twice), is off by under 80 u of its magnitude: 130 u of the
    magnitudes' sum.  A few rows weigh 64 times the others, the first and the last among them: without one of these some column is off by more."""
    from test_zzz_row_operators import block_inputs, cuda, norm_bwd_reference, norm_reference, wide
    eps, scale = 1e-6, 0.75
    r, f, ga, wp, wn, dr, dh = block_inputs(n, c, stream, dtype, gate, 21)
    for t in (dr, dh):                                 # rows that are the first and last of their rounds weigh more
        t[[0, 1, n // 2, n - 2, n - 1]] *= 64
    dev = cuda(dr, dh, r, f, ga, wp, wn)
    if packed:
        dev[3] = pcpp.pcpp_act_pack(dev[3])
        f = pcpp.pcpp_act_unpack(dev[3], F32)
    got = pcpp.pcpp_block_norm_bwd(*dev, post_norm=kind, pre_norm=kind, residual_scale=scale, eps=eps, dtype=dtype)
    r, f, ga, wp, wn, dr, dh = wide(r, f, ga, wp, wn, dr, dh)
    nr, rstd, mr = norm_reference(r, kind, eps, r.abs())
    y = wn * dh
    through, tmag = norm_bwd_reference(y, y.abs(), nr, mr, rstd, kind)
    d, dmag = dr + through, dr.abs() + tmag
    sigma, off = (torch.sigmoid(ga), 1 + ga.abs()) if ga is not None else (1.0, 1.0)
    nf, _, mf = norm_reference(f, kind, eps, f.abs())
    for what, terms, mags in (("dw_pre", dh * nr, dh.abs() * mr), ("dw_post", d * sigma * nf, dmag * sigma * off * mf)):
        off_by = (getattr(got, what).double().cpu() - terms.sum(0)).abs()
        bound = 130 * U * mags.sum(0)
        assert (off_by <= bound).all(), (what, float((off_by / bound).max()))
        for row in (0, n - 1):                         # a lost first or last row would be seen
            assert (terms[row].abs() > 2 * bound).any(), what
    again = pcpp.pcpp_block_norm_bwd(*dev, post_norm=kind, pre_norm=kind, residual_scale=scale, eps=eps, dtype=dtype)
    assert torch.equal(got.dw_pre, again.dw_pre) and torch.equal(got.dw_post, again.dw_post)
