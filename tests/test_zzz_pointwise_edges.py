"""The pointwise layers' operators where a batch has no rows, and where a single row lies anywhere."""
import pytest
import torch

from pointwise_reference import BF16, F32, U, activate
from test_zzz_pointwise import pcpp, rng, rows_of, within  # noqa: F401  (pcpp: the fixture)

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("c_out,c", [(1, 1), (40, 96), (130, 33), (300, 257)])
def test_gradients_of_no_rows(pcpp, c_out, c):
    """A batch without rows goes back as it went forward: sums of nothing."""
    dy, x = torch.empty(0, c_out, device="cuda"), torch.empty(0, c, dtype=BF16, device="cuda")
    d, h = pcpp.pcpp_mx_pack(dy, columns=True, random=rng(pcpp)), pcpp.pcpp_mx_pack(x, rows=False, columns=True)
    assert pcpp.pcpp_mx_unpack(h.columns).shape == (c, 0)
    dw = pcpp.pcpp_mx_product(d.columns, h.columns, dtype=F32)
    assert dw.shape == (c_out, c) and dw.dtype == F32 and not dw.any()
    weights = pcpp.pcpp_mx_pack(rows_of(c, c_out, F32)).rows
    assert pcpp.pcpp_mx_product(d.rows, weights).shape == (0, c)
    # ... with what stands behind a sum, into the middle of a tensor, and captured
    bias = rows_of(1, c, F32, 5)[0]
    wide = torch.full((c_out + 2, c), 7.0, device="cuda")
    call = lambda: pcpp.pcpp_mx_product(d.columns, h.columns, bias, act=pcpp.ACT_SILU, out=wide[1:-1])  # noqa: E731
    ref = activate(bias.double().cpu(), "silu").expand(c_out, c)
    within(call(), ref, 16 * U * (bias.double().cpu().abs() + ref.abs()), "bias")
    want = wide.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        wide[1:-1] = float("nan")
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(wide, want) and (wide[0] == 7).all() and (wide[-1] == 7).all()
    with pytest.raises((AssertionError, pcpp.PcppError)):
        pcpp.pcpp_mx_product(d.columns, pcpp.pcpp_mx_pack(rows_of(5, c, F32), rows=False, columns=True).columns)
    with pytest.raises((AssertionError, pcpp.PcppError)):
        pcpp.pcpp_mx_linear(torch.empty(3, 0, device="cuda"), h.columns)


@gpu
@pytest.mark.parametrize("m,k", [(1, 1), (300, 4096), (64, 64), (257, 1000), (33, 16_384), (33, 16_400)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("at", [1, 2, 3])
def test_one_row_at_any_address(pcpp, m, k, dtype, at):
    """The single token's linear layer on a row that starts between two wide loads: the same bits."""
    x, w, bias = rows_of(1, k, dtype, 51), pcpp.pcpp_mx_pack(rows_of(m, k, F32, 52, scale=k ** -0.5)).rows, rows_of(1, m, F32, 53)[0]
    wider = torch.full((1, k + 5), float("nan"), dtype=dtype, device="cuda")
    wider[:, at:at + k] = x
    row = wider[:, at:at + k]
    assert row.data_ptr() % 16 != 0
    y = pcpp.pcpp_mx_linear(x, w, bias, act=pcpp.ACT_GELU)
    assert torch.isfinite(y).all() and torch.equal(y, pcpp.pcpp_mx_linear(row, w, bias, act=pcpp.ACT_GELU))


@gpu
def test_every_output_that_is_given_is_written_and_counts(pcpp):
    x = rows_of(30, 64, F32)
    a, w = pcpp.pcpp_mx_pack(x).rows, pcpp.pcpp_mx_pack(rows_of(64, 64, F32)).rows
    for rows, call in ((30, lambda out: pcpp.pcpp_dropout_fwd(x, 0.5, rng(pcpp), out=out)), (30, lambda out: pcpp.pcpp_dropout_bwd(x, 0.5, rng(pcpp), out=out)),
                       (30, lambda out: pcpp.pcpp_group_norm_fwd(x, 4, out=out).y), (30, lambda out: pcpp.pcpp_mx_linear(x, w, out=out)),
                       (30, lambda out: pcpp.pcpp_mx_product(a, w, out=out)), (64, lambda out: pcpp.pcpp_mx_unpack(w, out=out))):
        out = torch.full((rows, 64), float("nan"), device="cuda")
        before = out._version
        y = call(out)
        assert y.data_ptr() == out.data_ptr() and out._version > before and torch.isfinite(out).all()
