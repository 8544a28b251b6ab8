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
