"""The pointwise layers' operators where a batch has no rows, offsets make no sense, a single row lies anywhere, a channel is constant; and which of the group norm's ways
through the rows each size takes.

The forward pass needs no workspace where a block takes a cloud from its statistics to its rows; by chunks it needs two numbers for every
chunk, cloud and group.  Chunks times groups past 4096 are joined by a launch of their own, others by the blocks that write y."""
import ctypes

import numpy as np
import pytest
import torch

from pointwise_reference import BF16, F32, U, activate, group_norm, group_norm_grads, slope
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


# ---- group norm by chunks ----------------------------------------------------------------------------------------

BY_CHUNKS = [  # n, c, groups, clouds, whether the chunks are joined by a launch of their own
    (9000, 16, 4, 2, False), (9000, 16, 4, 100, False), (9000, 91, 13, 3, False), (70_000, 64, 64, 2, True), (70_000, 64, 64, 70, True), (9000, 520, 260, 3, True),
]


def takes_chunks(lib, n, c, groups, clouds, launch):
    size = lib.pcpp_group_norm_workspace_bytes(n, c, clouds, groups, 0)
    assert size > 0                                    # 8 bytes for (chunks + clouds - 1) groups, and for clouds groups
    pairs = size // 8 - (2 * clouds - 1) * groups      # chunks times groups, up to 62 more for whole lines of 256 bytes
    assert pairs > 4096 + 62 if launch else pairs <= 4096


class Guarded:
    """Room of a caller's with a margin on both sides that nobody may write to."""

    def __init__(self, size, fill=0x5A):
        self.whole = torch.full((size + 1024,), fill, dtype=torch.uint8, device="cuda")
        self.size, self.fill = size, fill

    def __call__(self):
        return ctypes.c_void_p(self.whole.data_ptr() + 512)

    def inside(self, dtype=F32):
        return self.whole[512:512 + self.size].view(dtype)

    def untouched(self):
        return bool((self.whole[:512] == self.fill).all() and (self.whole[512 + self.size:] == self.fill).all())


class Norm:
    """Both directions through the C entry points, every output and workspace between margins."""

    def __init__(self, pcpp, x, groups, off):
        self.lib, self.x, self.off = pcpp.library(), x, off
        self.n, self.c, self.groups, self.clouds = *x.shape, groups, off.numel() - 1
        size = self.lib.pcpp_group_norm_workspace_bytes
        self.y, self.dx = Guarded(4 * x.numel()), Guarded(4 * x.numel())
        self.stats, self.dw, self.db = Guarded(8 * groups * self.clouds), Guarded(4 * self.c), Guarded(4 * self.c)
        self.rooms = [Guarded(size(self.n, self.c, self.clouds, groups, b)) for b in (0, 1)]
        self.all = [self.y, self.dx, self.stats, self.dw, self.db] + self.rooms

    def __call__(self, dy, act=0):
        at = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        rc = self.lib.pcpp_group_norm_fwd(at(self.x), self.c, None, None, at(self.off), self.clouds, self.groups, act, 1e-3, None, 0, 0.0, self.n, self.c, 0,
                                          self.y(), self.stats(), self.rooms[0](), self.rooms[0].size, stream)
        assert rc == 0, self.lib.pcpp_last_error()
        rc = self.lib.pcpp_group_norm_bwd(at(dy), at(self.x), self.c, self.stats(), None, None, at(self.off), self.clouds, self.groups, act, None, 0, 0.0,
                                          self.n, self.c, 0, self.dx(), self.dw(), self.db(), self.rooms[1](), self.rooms[1].size, stream)
        assert rc == 0, self.lib.pcpp_last_error()
        torch.cuda.synchronize()
        assert all(g.untouched() for g in self.all)
        y, dx, stats = self.y.inside().view(self.n, self.c), self.dx.inside().view(self.n, self.c), self.stats.inside().view(self.clouds, self.groups, 2)
        return y, stats, dx, self.dw.inside(), self.db.inside()


def spread(n, clouds):
    """Offsets of clouds of all sizes, some empty, the first row and the last of none."""
    cuts = np.sort(np.random.default_rng(clouds).integers(1, n, clouds + 1))
    cuts[clouds // 2] = cuts[clouds // 2 + 1]
    return [int(v) for v in cuts]


@gpu
@pytest.mark.parametrize("n,c,groups,clouds,launch", BY_CHUNKS)
def test_by_chunks(pcpp, n, c, groups, clouds, launch):
    """Values, and rows that belong to no cloud left as they were."""
    takes_chunks(pcpp.library(), n, c, groups, clouds, launch)
    offsets = spread(n, clouds)
    x, dy, off = rows_of(n, c, F32, 81), rows_of(n, c, F32, 82), torch.tensor(offsets, dtype=torch.int32, device="cuda")
    y, stats, dx, dw, db = Norm(pcpp, x, groups, off)(dy, pcpp.ACT_SILU)
    y_ref, stats_ref, off_y, off_stats = group_norm(x, groups, None, None, offsets, "silu", 1e-3, None)
    refs = group_norm_grads(dy, x, stats, None, None, offsets, "silu", None)
    lo, hi = offsets[0], offsets[-1]
    assert 0 < lo and hi < n
    within(stats, stats_ref, off_stats, "mean_rstd")
    within(y[lo:hi], y_ref[lo:hi], off_y[lo:hi], "y")
    within(dx[lo:hi], refs[0][0][lo:hi], refs[0][1][lo:hi], "dx")
    within(dw, *refs[1], "dw")
    within(db, *refs[2], "db")
    for t in (y, dx):
        left = torch.cat([t[:lo], t[hi:]])
        assert (left.contiguous().view(torch.uint8) == 0x5A).all()


@gpu
@pytest.mark.parametrize("n,c,groups,clouds,launch", BY_CHUNKS)
def test_by_chunks_offsets_that_make_no_sense_stay_inside(pcpp, n, c, groups, clouds, launch):
    """Every output and both workspaces have margins; entries outside the tensor are its ends."""
    takes_chunks(pcpp.library(), n, c, groups, clouds, launch)
    x, dy = rows_of(n, c, F32, 83), rows_of(n, c, F32, 84)
    least, most = -2 ** 31, 2 ** 31 - 1
    g = np.random.default_rng(85)
    ordered = spread(n, clouds)
    orders = [ordered[::-1], [most] + [least] * clouds, [most, least] * (clouds // 2) + [5] * (1 + clouds % 2), [n] * (clouds + 1), [least] * (clouds + 1),
              g.integers(least, most, clouds + 1).tolist(), g.integers(-n, 2 * n, clouds + 1).tolist(), g.permutation(ordered).tolist()]
    for offsets in orders:
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        assert off.numel() == clouds + 1
        Norm(pcpp, x, groups, off)(dy)
        pcpp.pcpp_dropout_fwd(x, 0.5, rng(pcpp), scope=pcpp.DROP_CLOUDS, offsets=off)
    torch.cuda.synchronize()
    outside = [least] + ordered[1:-1] + [most]
    inside = [0] + ordered[1:-1] + [n]
    got, want = (Norm(pcpp, x, groups, torch.tensor(o, dtype=torch.int32, device="cuda"))(dy) for o in (outside, inside))
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("n,c,groups,clouds,launch", BY_CHUNKS)
def test_by_chunks_infinities_stay_in_their_cloud_and_group(pcpp, n, c, groups, clouds, launch):
    takes_chunks(pcpp.library(), n, c, groups, clouds, launch)
    offsets = [0] + spread(n, clouds)[1:-1] + [n]
    x, dy, width = rows_of(n, c, F32, 86), rows_of(n, c, F32, 87), c // groups
    bad = torch.zeros(n, c, dtype=torch.bool)
    channels = torch.zeros(c, dtype=torch.bool)
    for cloud, group, value in ((0, groups - 1, float("inf")), (clouds - 1, 1, float("nan")), (clouds - 1, 0, float("-inf"))):
        lo, hi = offsets[cloud], offsets[cloud + 1]
        assert lo < hi
        x[(lo + hi) // 2, group * width] = value
        bad[lo:hi, group * width:(group + 1) * width] = True
        channels[group * width:(group + 1) * width] = True
    y, stats, dx, dw, db = (t.cpu() for t in Norm(pcpp, x, groups, torch.tensor(offsets, dtype=torch.int32, device="cuda"))(dy))
    for t in (y, dx):
        assert torch.isnan(t[bad]).all() and torch.isfinite(t[~bad]).all()
    assert torch.isnan(dw[channels]).all() and torch.isfinite(dw[~channels]).all() and torch.isfinite(db).all()


@gpu
@pytest.mark.parametrize("n,c,groups,clouds,launch", BY_CHUNKS)
def test_by_chunks_clouds_without_a_row(pcpp, n, c, groups, clouds, launch):
    takes_chunks(pcpp.library(), n, c, groups, clouds, launch)
    x, off = rows_of(n, c, F32, 88), torch.full((clouds + 1,), 100, dtype=torch.int32, device="cuda")
    y, stats, dx, dw, db = Norm(pcpp, x, groups, off)(x)
    assert not stats.any() and not dw.any() and not db.any()
    for t in (y, dx):
        assert (t.view(torch.uint8) == 0x5A).all()


# ---- channels that are the same in every row ---------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("n,c,offsets", [(40, 24, [0, 1, 2, 17, 40]), (60, 5, None), (9000, 16, [0, 4000, 9000]), (9000, 91, [0, 1, 9000]), (900, 1023, [0, 300, 900]),
                                         (70_000, 64, [0, 35_000, 70_000])])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_constant_channels(pcpp, n, c, offsets, dtype, act):
    """Groups of one channel that a cloud's rows all share, from 1 to 3e5: x - mean is zero without a rounding, so y is act(b), dw is zero and dx has no
    share of v, however small eps is beside the numbers."""
    g = torch.Generator().manual_seed(91)
    w, b = (1 + 0.3 * torch.randn(c, generator=g)).cuda(), (0.3 * torch.randn(c, generator=g)).cuda()
    ranges = [(0, n)] if offsets is None else list(zip(offsets[:-1], offsets[1:]))
    x, dy = torch.empty(n, c, dtype=dtype), rows_of(n, c, dtype, 92)
    for lo, hi in ranges:
        x[lo:hi] = (torch.exp(12.6 * torch.rand(1, c, generator=g)) * torch.sign(torch.randn(1, c, generator=g))).to(dtype)
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    code = {"none": pcpp.ACT_NONE, "silu": pcpp.ACT_SILU}[act]
    eps, rstd = 1e-5, float(np.float32(1e-5)) ** -0.5
    y = pcpp.pcpp_group_norm_fwd(x.cuda(), c, w, b, off, act=code, eps=eps)
    z = b.double().cpu()
    ref = activate(z, act).expand(n, c)
    within(y.y, ref, 16 * U * (z.abs() + ref.abs()), "y")
    d = pcpp.pcpp_group_norm_bwd(dy, x.cuda(), y.mean_rstd, w, b, off, act=code)
    assert not d.dw.any()
    dz = dy.double().cpu() * slope(z, act)
    for lo, hi in ranges:
        depth, t = 64 + (hi - lo) / 32, w.double().cpu() * dz[lo:hi]
        m1 = t.mean(0)
        bound = rstd * (16 * U * (t.abs() + m1.abs() + (w.double().cpu() * dy[lo:hi].double().cpu()).abs()) + (depth + 16) * U * t.abs().mean(0))
        within(d.dx[lo:hi], rstd * (t - m1), bound, "dx")
