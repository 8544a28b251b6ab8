"""The pointwise layers' operators against plain 64-bit forms: random numbers by counter and dropout, group norm with an activation and its
gradients, rows in 4 bits and their products; and a run of them together, eager and in a captured graph.

Tolerances.  fp32 results are held to the bounds that the references derive from u = 2^-24 and the depth of the kernels' sums; a result in
bf16 may be off by its own rounding, 2^-8 of it, too.  What has no rounding (masks, codes, 4-bit values) has to be equal."""
import numpy as np
import pytest
import torch

from pointwise_reference import (BF16, F32, U, activate, bounds_of, factors, from_bits, group_norm, group_norm_grads, philox, slope, to_bits,
                                 uniform16)

gpu = pytest.mark.gpu
SEED, STEP = 0x123456789ABCDEF, 77


@pytest.fixture(scope="module")
def pcpp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_23227_amd as m
    m.library()
    return m


def rng(pcpp, site=3, seed=SEED, step=STEP):
    return pcpp.Random(torch.tensor([seed, step], device="cuda"), site)


def within(got, ref, off, what):
    """|got - ref| <= off, and half a unit of bf16 more for a bf16 result; infinities and NaN have no place here."""
    tol = off + (2.0 ** -8 * (ref.abs() + off) if got.dtype == BF16 else 2.0 ** -23 * ref.abs())
    got = got.double().cpu()
    assert got.shape == ref.shape and torch.isfinite(got).all(), what
    worst = float(((got - ref).abs() - tol).max()) if got.numel() else 0.0
    assert worst <= 1e-38, (what, worst, float((got - ref).abs().max()))


def rows_of(n, c, dtype, seed=0, pitch=0, scale=1.0, mean=0.5):
    """[n, c], of wider rows where a pitch is given."""
    g = torch.Generator().manual_seed(seed)
    x = ((torch.randn(n, c, generator=g) + mean * torch.randn(1, c, generator=g)) * scale).to(dtype)
    if not pitch:
        return x.cuda()
    wide = torch.full((n, c + pitch), float("nan"), dtype=dtype, device="cuda")
    wide[:, 1:1 + c] = x.cuda()
    return wide[:, 1:1 + c]


# ---- random numbers ----------------------------------------------------------------------------------------------

def test_reference_numbers():
    """The published known answers of ten rounds of Philox 4x32."""
    hexes = lambda *v: np.array(v, np.uint64)  # noqa: E731
    assert (philox(hexes(0, 0, 0, 0), (0, 0)) == hexes(0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)).all()
    ones = 0xFFFFFFFF
    assert (philox(hexes(ones, ones, ones, ones), (ones, ones)) == hexes(0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)).all()
    u = uniform16(SEED, STEP, 1, 4000, 20)
    assert abs(u.mean() / 65535 - 0.5) < 0.01 and abs(np.corrcoef(u[:, 0], u[:, 1])[0, 1]) < 0.06


@gpu
@pytest.mark.parametrize("n,c,pitch", [(1, 1, 0), (1, 8, 0), (3, 7, 0), (5, 9, 0), (33, 91, 0), (700, 33, 6), (64, 256, 3), (129, 64, 0), (3, 65536, 0), (0, 16, 0)])
@pytest.mark.parametrize("dtype,stream", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("p", [0.1, 0.0, 1.0])
def test_dropout(pcpp, n, c, pitch, dtype, stream, p):
    x, random = rows_of(n, c, dtype, 1, pitch), rng(pcpp)
    k = torch.from_numpy(factors(uniform16(SEED, STEP, 3, n, c), p))
    branch = k * x.double().cpu()
    for residual in (None, rows_of(n, c, stream, 2)):
        r = 0.0 if residual is None else residual.double().cpu()
        if residual is None and stream != dtype:
            continue
        y = pcpp.pcpp_dropout_fwd(x, p, random, residual)
        assert y.dtype == stream
        within(y, r + branch, 2 * U * (branch.abs() + abs(r)), "y")
    dy = rows_of(n, c, stream, 3)
    dx = pcpp.pcpp_dropout_bwd(dy, p, random, dtype=dtype)
    assert dx.dtype == dtype
    within(dx, k * dy.double().cpu(), U * (k * dy.double().cpu()).abs(), "dx")
    assert ((dx != 0).cpu() == (k * dy.double().cpu() != 0)).all()


@gpu
@pytest.mark.parametrize("c", [5, 64, 91])
def test_dropout_of_rows_and_clouds(pcpp, c):
    n, random = 500, rng(pcpp, 9, step=-1)             # (a step of all ones)
    x, residual = rows_of(n, c, BF16, 4), rows_of(n, c, F32, 5)
    kept = factors(uniform16(SEED, -1, 9, n, 1), 0.5)
    assert 0 < (kept > 0).sum() < n
    y = pcpp.pcpp_dropout_fwd(x, 0.5, random, residual, scope=pcpp.DROP_ROWS)
    within(y, residual.double().cpu() + torch.from_numpy(kept) * x.double().cpu(), 4 * U * (residual.abs() + 2 * x.abs()).double().cpu(), "rows")
    # clouds: empty ones, rows before the first and behind the last
    offsets = torch.tensor([7, 7, 100, 101, 101, 300, 480], dtype=torch.int32)
    kept = factors(uniform16(SEED, -1, 9, 6, 1), 0.5)[:, 0]
    out = torch.full((n, c), 5.0, device="cuda")
    y = pcpp.pcpp_dropout_fwd(x, 0.5, random, residual, scope=pcpp.DROP_CLOUDS, offsets=offsets.cuda(), out=out)
    ref = torch.full((n, c), 5.0, dtype=torch.float64)
    for b, (lo, hi) in enumerate(bounds_of(offsets, n)):
        ref[lo:hi] = residual[lo:hi].double().cpu() + kept[b] * x[lo:hi].double().cpu()
    within(y, ref, 4 * U * (residual.abs() + 2 * x.abs()).double().cpu(), "clouds")
    assert y.data_ptr() == out.data_ptr()
    dx = pcpp.pcpp_dropout_bwd(residual, 0.5, random, scope=pcpp.DROP_CLOUDS, offsets=offsets.cuda(), dtype=BF16, out=torch.full((n, c), 5.0, dtype=BF16, device="cuda"))
    for b, (lo, hi) in enumerate(bounds_of(offsets, n)):
        ref[lo:hi] = kept[b] * residual[lo:hi].double().cpu()
    within(dx, ref, 2 * U * ref.abs(), "clouds' gradient")


@gpu
def test_dropout_leaves_nothing_of_what_it_drops(pcpp):
    x = torch.full((64, 24), float("inf"), device="cuda")
    x[:, ::2] = float("nan")
    y = pcpp.pcpp_dropout_fwd(x, 0.5, rng(pcpp))
    kept = torch.from_numpy(factors(uniform16(SEED, STEP, 3, 64, 24), 0.5) > 0)
    assert (y.cpu()[~kept] == 0).all() and not torch.isfinite(y.cpu()[kept]).any()
    y = pcpp.pcpp_dropout_fwd(x, 1.0, rng(pcpp), torch.ones_like(x))
    assert (y == 1).all()


# ---- group norm --------------------------------------------------------------------------------------------------

NORMS = [  # n, c, groups, offsets, act, p, pitch
    (1, 1, 1, None, "none", 0.0, 0), (1, 256, 32, None, "silu", 0.0, 0), (3, 256, 32, None, "gelu", 0.0, 0), (7, 5, 5, None, "relu", 0.3, 0),
    (300, 7, 1, [0, 0, 100, 101, 300], "silu", 0.25, 0), (500, 91, 13, [0, 1, 300, 300, 499], "gelu", 0.1, 5), (40, 9, 3, [3, 30], "none", 0.5, 0),
    (1500, 64, 8, [0, 700, 1500], "silu", 0.1, 0), (2000, 64, 64, None, "gelu", 0.0, 3), (900, 520, 4, [10, 450, 880], "silu", 0.2, 0),
    (700, 1021, 1, None, "gelu", 0.1, 0), (600, 1024, 1024, [0, 599, 600], "none", 0.0, 0), (1300, 33, 11, [0, 1300], "silu", 0.1, 0),
    (2500, 16, 2, [0] + list(range(0, 2500, 31)) + [2500], "gelu", 0.1, 0), (5000, 3, 1, None, "relu", 0.0, 0),
    (400, 32, 4, [100, 100, 100], "silu", 0.0, 0),     # no cloud has a row
    (130, 256, 32, [0, 0, 5, 60, 130], "gelu", 0.1, 0), (900, 40, 5, [0] + list(range(2, 900, 9)), "silu", 0.1, 3),    # a block to a cloud
    (3000, 40, 5, [1] + list(range(4, 3000, 11)) + [2999], "gelu", 0.2, 0),    # short chunks for short clouds
]


@gpu
@pytest.mark.parametrize("n,c,groups,offsets,act,p,pitch", NORMS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_group_norm(pcpp, n, c, groups, offsets, act, p, pitch, dtype):
    x = rows_of(n, c, dtype, 11, pitch)
    g = torch.Generator().manual_seed(12)
    w, b = (1 + 0.3 * torch.randn(c, generator=g)).cuda(), (0.3 * torch.randn(c, generator=g)).cuda()
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    factor = factors(uniform16(SEED, STEP, 3, n, c), p) if p else None
    acts = {"none": pcpp.ACT_NONE, "relu": pcpp.ACT_RELU, "silu": pcpp.ACT_SILU, "gelu": pcpp.ACT_GELU}
    how = dict(act=acts[act], p=p, random=rng(pcpp) if p else None)
    inside = torch.zeros(n, dtype=torch.bool)
    for lo, hi in bounds_of(offsets, n):
        inside[lo:hi] = True
    for weights in ((w, b), (None, None)):
        y_ref, stats, off_y, off_stats = group_norm(x, groups, *weights, offsets, act, 1e-3, factor)
        out = torch.full((n, c), 9.0, dtype=dtype, device="cuda")
        y = pcpp.pcpp_group_norm_fwd(x, groups, *weights, off, eps=1e-3, out=out, **how)
        assert y.y.data_ptr() == out.data_ptr() and (out.cpu()[~inside] == 9).all()
        within(out.cpu()[inside], y_ref[inside], off_y[inside], "y")
        within(y.mean_rstd, stats, off_stats, "mean_rstd")
        again = pcpp.pcpp_group_norm_fwd(x, groups, *weights, off, eps=1e-3, statistics=False, out=torch.zeros_like(out), **how)
        assert again.mean_rstd is None and torch.equal(again.y.cpu()[inside], out.cpu()[inside])
        # gradients, from statistics that are inputs; z of a relu stays off its corner
        dy = rows_of(n, c, dtype, 13)
        xs, ws, given = x, weights, y.mean_rstd
        if act == "relu":
            xs = (torch.randint(-6, 7, (n, c), generator=g) * 0.5).to(dtype).cuda()
            ws, given = (torch.ones_like(w), torch.full_like(b, 0.25)), torch.stack([torch.zeros(stats.shape[:2]), torch.ones(stats.shape[:2])], 2).cuda()
        d = pcpp.pcpp_group_norm_bwd(dy, xs, given, *ws, off, **how)
        refs = group_norm_grads(dy, xs, given, *ws, offsets, act, factor)
        within(d.dx.cpu()[inside], refs[0][0][inside], refs[0][1][inside], "dx")
        within(d.dw, *refs[1], "dw")
        within(d.db, *refs[2], "db")
        only = pcpp.pcpp_group_norm_bwd(dy, xs, given, *ws, off, of_x=False, **how)
        assert only.dx is None and torch.equal(only.dw, d.dw) and torch.equal(only.db, d.db)
        only = pcpp.pcpp_group_norm_bwd(dy, xs, given, *ws, off, of_weights=False, **how)
        assert only.dw is None and only.db is None and torch.equal(only.dx.cpu()[inside], d.dx.cpu()[inside])


@gpu
@pytest.mark.parametrize("n,c,groups,offsets,act", [(40, 24, 4, [0, 17, 40], "silu"), (900, 24, 3, [0, 400, 900], "gelu")])
def test_group_norm_gradients_are_those_of_its_formula(pcpp, n, c, groups, offsets, act):
    """The 64-bit gradients against differences of the 64-bit forward pass, and automatic differentiation of it."""
    x, w, b = rows_of(n, c, F32, 21).double().cpu(), rows_of(1, c, F32, 22)[0].double().cpu(), rows_of(1, c, F32, 23)[0].double().cpu()
    dy = rows_of(n, c, F32, 24).double().cpu()
    f = lambda x, w, b: (group_norm(x, groups, w, b, offsets, act, 1e-3, None)[0] * dy).sum()  # noqa: E731
    stats = group_norm(x, groups, w, b, offsets, act, 1e-3, None)[1]
    (dx, _), (dw, _), (db, _) = group_norm_grads(dy, x, stats, w, b, offsets, act, None)
    g = torch.Generator().manual_seed(25)
    for i, (grad, args) in enumerate(((dx, x), (dw, w), (db, b))):
        way = torch.randn(args.shape, generator=g, dtype=torch.float64)
        h = 1e-5
        moved = [[a + s * h * way if j == i else a for j, a in enumerate((x, w, b))] for s in (1, -1)]
        slope_ = (f(*moved[0]) - f(*moved[1])) / (2 * h)
        assert abs(float(slope_ - (grad * way).sum())) < 1e-6 * float((grad * way).abs().sum())


@gpu
def test_group_norm_far_from_zero(pcpp):
    """A mean of a thousand deviations: the statistics lose no more than the inputs' own rounding does."""
    x = (1000.0 + torch.randn(3000, 32, generator=torch.Generator().manual_seed(1))).cuda()
    y = pcpp.pcpp_group_norm_fwd(x, 4, eps=1e-6)
    ref, stats, off, off_stats = group_norm(x, 4, None, None, None, "none", 1e-6, None)
    within(y.mean_rstd, stats, off_stats, "mean_rstd")
    within(y.y, ref, off, "y")


@gpu
def test_group_norm_keeps_infinities_to_their_group(pcpp):
    x = rows_of(1000, 32, F32, 31)
    x[500, 9], x[20, 30] = float("inf"), float("nan")
    off = torch.tensor([0, 100, 700, 1000], dtype=torch.int32, device="cuda")
    y = pcpp.pcpp_group_norm_fwd(x, 4, None, None, off)
    bad = torch.zeros(1000, 32, dtype=torch.bool)
    bad[100:700, 8:16] = bad[:100, 24:] = True
    assert torch.isnan(y.y.cpu()[bad]).all() and torch.isfinite(y.y.cpu()[~bad]).all()
    dy = rows_of(1000, 32, F32, 32)
    d = pcpp.pcpp_group_norm_bwd(dy, x, y.mean_rstd, None, None, off)
    assert torch.isnan(d.dx.cpu()[bad]).all() and torch.isfinite(d.dx.cpu()[~bad]).all()


@gpu
def test_group_norm_of_thousands_of_clouds(pcpp):
    """... found by three loads of 64 offsets, and of no rows at all."""
    n, c, offsets = 9000, 6, [0, 0] + list(range(1, 8998, 2)) + [8997, 8999]
    x, dy, off = rows_of(n, c, F32, 35), rows_of(n, c, F32, 36), torch.tensor(offsets, dtype=torch.int32, device="cuda")
    y_ref, stats, off_y, off_stats = group_norm(x, 3, None, None, offsets, "silu", 1e-3, None)
    y = pcpp.pcpp_group_norm_fwd(x, 3, None, None, off, act=pcpp.ACT_SILU, eps=1e-3)
    within(y.mean_rstd, stats, off_stats, "mean_rstd")
    within(y.y[:8999], y_ref[:8999], off_y[:8999], "y")
    d = pcpp.pcpp_group_norm_bwd(dy, x, y.mean_rstd, None, None, off, act=pcpp.ACT_SILU)
    dx, dw, db = group_norm_grads(dy, x, y.mean_rstd, None, None, offsets, "silu", None)
    within(d.dx[:8999], dx[0][:8999], dx[1][:8999], "dx")
    within(d.dw, *dw, "dw")
    within(d.db, *db, "db")
    none = torch.zeros(len(offsets), dtype=torch.int32, device="cuda")
    y = pcpp.pcpp_group_norm_fwd(x[:0], 3, None, None, none)
    d = pcpp.pcpp_group_norm_bwd(dy[:0], x[:0], y.mean_rstd, None, None, none)
    assert y.y.shape == (0, 6) and not y.mean_rstd.any() and not d.dw.any() and not d.db.any()


@gpu
def test_offsets_that_make_no_sense_stay_inside(pcpp):
    """Offsets outside the tensor count as its ends: the calls neither fault nor write elsewhere."""
    n, c = 800, 16
    wide = torch.full((n + 64, c), 3.0, device="cuda")
    x, out = rows_of(n, c, F32, 33), wide[32:n + 32]
    for bad in ([-5, 10, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 5], [700, 300, 900]):
        off = torch.tensor(bad, dtype=torch.int32, device="cuda")
        y = pcpp.pcpp_group_norm_fwd(x, 4, None, None, off, out=out)
        pcpp.pcpp_group_norm_bwd(x, x, y.mean_rstd, None, None, off)
        pcpp.pcpp_dropout_fwd(x, 0.5, rng(pcpp), scope=pcpp.DROP_CLOUDS, offsets=off, out=out)
        torch.cuda.synchronize()
        assert (wide[:32] == 3).all() and (wide[n + 32:] == 3).all()


# ---- rows in 4 bits ----------------------------------------------------------------------------------------------

def special(n, c, dtype, seed=41):
    """Rows with zeros, ties, borders between powers, tiny and huge numbers, infinities and NaN."""
    g = np.random.default_rng(seed)
    x = g.standard_normal((n, c)) * np.exp2(g.integers(-6, 6, (n, 1)))
    if n >= 24:
        x[1] = 0.0
        x[2] = np.exp2(-140.0) * g.standard_normal(c)
        x[3] = 3.3e38 * np.sign(x[3])
        x[4] = np.resize(np.array([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -2.5, -5, 0.5, -0.0, 1]), c)
        x[5] = np.resize(np.array([7, 6.99, 1, -3]), c)
        x[6] = np.resize(np.array([6.98, -1, 0.2]), c)
        x[7, c // 2], x[8, 0], x[9, c - 1] = np.inf, np.nan, -np.inf
        x[10] = np.resize(np.array([6.0000005, 4, 1]), c)
        x[11] = 2.0 ** -126 * np.resize(np.array([6, 7, 0.3, 0.25]), c)
    return torch.from_numpy(x).to(dtype)


SIZES = [(1, 1), (1, 32), (3, 33), (40, 91), (30, 128), (200, 20), (129, 64), (500, 65), (33, 1000), (257, 256), (24, 7), (2, 8192)]


@gpu
@pytest.mark.parametrize("n,c", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("at_random", [False, True])
def test_pack(pcpp, n, c, dtype, at_random):
    x = special(n, c, dtype)
    u = uniform16(SEED, STEP, 6, n, c) if at_random else None
    random = rng(pcpp, 6) if at_random else None
    wide = torch.full((n, c + 3), float("nan"), dtype=dtype, device="cuda")
    wide[:, 2:2 + c] = x.cuda()
    ref = {"rows": to_bits(x.double().numpy(), u), "columns": to_bits(x.double().numpy().T, None if u is None else u.T)}
    for src in (x.cuda(), wide[:, 2:2 + c]):
        for rows, columns in ((True, False), (False, True), (True, True)):
            m = pcpp.pcpp_mx_pack(src, rows=rows, columns=columns, random=random)
            assert (m.rows is not None, m.columns is not None) == (rows, columns)
            for name, got in (("rows", m.rows), ("columns", m.columns)):
                if got is None:
                    continue
                q, scales, values = ref[name]
                assert got.c == values.shape[1]
                assert (got.scales.cpu().numpy() == scales).all(), name
                assert (got.q.cpu().numpy() == q).all(), name
                for out in (BF16, F32):
                    v = pcpp.pcpp_mx_unpack(got, out).double().cpu().numpy()
                    assert v.shape == values.shape and ((v == values) | (np.isnan(v) & np.isnan(values))).all()


@gpu
def test_unpack_takes_any_scale(pcpp):
    """All codes with all scales that 32 bits hold the values of, the smallest among them (2^-127)."""
    scales = np.zeros((256, 4), np.uint8)
    scales[:, 0] = np.arange(256)
    q = np.tile(np.arange(16, dtype=np.uint8) | (np.arange(16, dtype=np.uint8)[::-1] << 4), (256, 1))
    m = pcpp.MxRows(torch.from_numpy(q).cuda(), torch.from_numpy(scales).cuda(), 32)
    ref = from_bits(q, scales, 32)
    for dtype in (BF16, F32):
        v = pcpp.pcpp_mx_unpack(m, dtype).double().cpu().numpy()
        fine = np.abs(ref) < 2.0 ** 128
        assert (v[fine] == ref[fine]).all() and np.isnan(v[255]).all() and np.isinf(v[253:255][~fine[253:255]]).all()


@gpu
def test_rounding_at_random_is_unbiased(pcpp):
    """The mean over many rows of one number: its value, within five deviations of the draws."""
    n = 20000
    x = torch.tensor([6.0, 0.1, 0.7, 1.9, 2.3, 3.3, 4.5, 5.9]).repeat(n, 4).cuda()
    v = pcpp.pcpp_mx_unpack(pcpp.pcpp_mx_pack(x, random=rng(pcpp)).rows, F32).double()
    gap = torch.tensor([0.0, 0.5, 0.5, 0.5, 1.0, 1.0, 2.0, 2.0]).repeat(4).double()
    off = (v.mean(0).cpu() - x[0].double().cpu()).abs()
    assert (off <= 5 * 0.5 * gap / n ** 0.5 + 2.0 ** -16 * gap + 1e-12).all()


def product_reference(a, b, bias, act):
    """(value, bound) of act(a b^T + bias): fp32 sums of depth k / 32 + 64, whatever their order."""
    y, size = a @ b.T, a.abs() @ b.abs().T
    off = (a.shape[1] / 32 + 64) * U * size
    if bias is not None:
        y, off = y + bias, off + U * (size + bias.abs())
    out = activate(y, act)
    return out, 1.13 * off + 16 * U * (y.abs() + out.abs())


PRODUCTS = [  # n, m, k
    (1, 1, 1), (1, 64, 64), (1, 300, 4096), (2, 257, 1000), (16, 128, 256), (17, 130, 129), (100, 91, 91), (128, 128, 128), (129, 255, 513), (300, 200, 31),
    (1000, 64, 32), (33, 1000, 2048), (512, 512, 512), (5, 3, 100_000), (91, 64, 33_333), (700, 520, 1500), (3500, 3601, 1100), (13, 40, 20_000),
    (16, 2100, 600), (9, 33, 16_384), (9, 33, 8192), (9, 33, 8193), (17, 70, 8000),
    (1, 40, 16_384), (1, 33, 16_400), (8, 24, 2048), (9, 24, 2048),
    (130, 256, 256), (130, 257, 256), (300, 100, 7), (129, 200, 257), (1000, 72, 91), (17, 9, 1),
]


@gpu
@pytest.mark.parametrize("n,m,k", PRODUCTS)
@pytest.mark.parametrize("dtype,act,biased", [(F32, "none", False), (BF16, "gelu", True), (F32, "silu", True), (BF16, "relu", False)])
def test_product_and_linear(pcpp, n, m, k, dtype, act, biased):
    x, w = rows_of(n, k, dtype, 51), rows_of(m, k, F32, 52, scale=k ** -0.5)
    bias = rows_of(1, m, F32, 53)[0] if biased else None
    acts = {"none": pcpp.ACT_NONE, "relu": pcpp.ACT_RELU, "silu": pcpp.ACT_SILU, "gelu": pcpp.ACT_GELU}
    packed, weights = pcpp.pcpp_mx_pack(x).rows, pcpp.pcpp_mx_pack(w).rows
    a, b = (pcpp.pcpp_mx_unpack(v, F32).double().cpu() for v in (packed, weights))
    ref, off = product_reference(a, b, None if bias is None else bias.double().cpu(), act)
    wide = torch.full((n + 2, m), 7.0, dtype=dtype, device="cuda")
    y = pcpp.pcpp_mx_product(packed, weights, bias, act=acts[act], out=wide[1:n + 1])
    within(y, ref, off, "product")
    assert (wide[0] == 7).all() and (wide[n + 1] == 7).all()
    z = pcpp.pcpp_mx_linear(x, weights, bias, act=acts[act])
    within(z, ref, off, "linear")
    wider = torch.full((n, k + 5), float("nan"), dtype=dtype, device="cuda")
    wider[:, 3:3 + k] = x
    assert torch.equal(z, pcpp.pcpp_mx_linear(wider[:, 3:3 + k], weights, bias, act=acts[act])) or n == 1


@gpu
@pytest.mark.parametrize("n,m,k", [(40, 70, 200), (200, 300, 512), (1, 40, 3000)])
def test_a_row_that_is_not_finite_stays_alone(pcpp, n, m, k):
    x, w = rows_of(n, k, F32, 54), rows_of(m, k, F32, 55)
    x[n - 1, k // 3] = float("inf")
    w[m // 2, 5] = float("nan")
    y = pcpp.pcpp_mx_linear(x, pcpp.pcpp_mx_pack(w).rows).cpu()
    bad = torch.zeros(n, m, dtype=torch.bool)
    bad[n - 1], bad[:, m // 2] = True, True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()


@gpu
def test_products_take_no_scale_from_behind_a_row(pcpp):
    """Scales past a row's last block may hold anything."""
    x, w = rows_of(20, 40, F32, 56), rows_of(24, 40, F32, 57)
    a, b = pcpp.pcpp_mx_pack(x).rows, pcpp.pcpp_mx_pack(w).rows
    y = pcpp.pcpp_mx_product(a, b, dtype=F32)
    a.scales[:, 2:], b.scales[:, 2:] = 255, 255
    assert torch.equal(y, pcpp.pcpp_mx_product(a, b, dtype=F32))


@gpu
@pytest.mark.parametrize("n", [0])
def test_no_rows(pcpp, n):
    x = torch.empty(0, 48, device="cuda")
    w = pcpp.pcpp_mx_pack(rows_of(16, 48, F32)).rows
    assert pcpp.pcpp_mx_linear(x, w).shape == (0, 16) and pcpp.pcpp_mx_unpack(pcpp.pcpp_mx_pack(x).rows).shape == (0, 48)
    y = pcpp.pcpp_group_norm_fwd(x, 4)
    assert y.y.shape == (0, 48) and (y.mean_rstd == 0).all()
    d = pcpp.pcpp_group_norm_bwd(x, x, y.mean_rstd)
    assert (d.dw == 0).all() and (d.db == 0).all()
    assert pcpp.pcpp_dropout_fwd(x, 0.5, rng(pcpp)).shape == (0, 48)


@gpu
def test_what_the_calls_refuse(pcpp):
    x, w = rows_of(20, 64, F32), pcpp.pcpp_mx_pack(rows_of(16, 64, F32)).rows
    r = rng(pcpp)
    refused = (AssertionError, TypeError, pcpp.PcppError)
    for call in (lambda: pcpp.pcpp_dropout_fwd(x.cpu(), 0.5, r), lambda: pcpp.pcpp_dropout_fwd(x, 0.5, None), lambda: pcpp.pcpp_dropout_fwd(x, 2.0, r),
                 lambda: pcpp.pcpp_dropout_fwd(x.half(), 0.5, r), lambda: pcpp.pcpp_dropout_fwd(x, 0.5, r, x[:10]), lambda: pcpp.pcpp_dropout_fwd(x, 0.5, r, x, out=x),
                 lambda: pcpp.pcpp_dropout_fwd(x.t(), 0.5, r), lambda: pcpp.pcpp_dropout_fwd(x, 0.5, pcpp.Random(r.state.int(), 0)),
                 lambda: pcpp.pcpp_dropout_fwd(x, 0.5, pcpp.Random(r.state, -1)), lambda: pcpp.pcpp_dropout_fwd(x, 0.5, r, scope=pcpp.DROP_CLOUDS, offsets=r.state),
                 lambda: pcpp.pcpp_group_norm_fwd(x, 5), lambda: pcpp.pcpp_group_norm_fwd(x, 0), lambda: pcpp.pcpp_group_norm_fwd(x, 4, x[0, :32]),
                 lambda: pcpp.pcpp_group_norm_fwd(x, 4, p=0.5), lambda: pcpp.pcpp_group_norm_fwd(x, 4, eps=0.0), lambda: pcpp.pcpp_group_norm_fwd(x, 4, out=x),
                 lambda: pcpp.pcpp_group_norm_bwd(x, x, torch.zeros(2, 4, 2, device="cuda")), lambda: pcpp.pcpp_group_norm_bwd(x, x.bfloat16(), torch.zeros(1, 4, 2, device="cuda")),
                 lambda: pcpp.pcpp_mx_pack(x, rows=False), lambda: pcpp.pcpp_mx_pack(x.double()), lambda: pcpp.pcpp_mx_unpack(pcpp.MxRows(w.q, w.scales, 65)),
                 lambda: pcpp.pcpp_mx_linear(x[:, :63], w), lambda: pcpp.pcpp_mx_linear(x, w, x[0]), lambda: pcpp.pcpp_mx_linear(x, w, act=9),
                 lambda: pcpp.pcpp_mx_product(w, pcpp.pcpp_mx_pack(x[:, :32]).rows), lambda: pcpp.pcpp_mx_product(w, w, out=x), lambda: pcpp.pcpp_mx_linear(x[:16, :16], pcpp.pcpp_mx_pack(x[:16, :16]).rows, out=x.view(-1)[:256].view(16, 16)),
                 lambda: pcpp.pcpp_mx_linear(x[:1], pcpp.pcpp_mx_pack(rows_of(64, 64, F32)).rows, out=x[:1])):
        with pytest.raises(refused):
            call()


# ---- together ----------------------------------------------------------------------------------------------------

class Layer:
    """One pointwise layer of a training step: norm, activation, dropout, a linear layer in 4 bits, dropout onto the residual; and back."""

    def __init__(self, pcpp, n=700, c=96, c_out=96, dtype=BF16):
        self.p, self.n, self.c, self.c_out, self.dtype = pcpp, n, c, c_out, dtype
        self.groups = 8 if c % 8 == 0 else 7
        self.x, self.residual, self.dy = rows_of(n, c, dtype, 61), rows_of(n, c_out, F32, 62), rows_of(n, c_out, F32, 63)
        self.w, self.b = 1 + rows_of(1, c, F32, 64)[0] * 0.1, rows_of(1, c, F32, 65)[0] * 0.1
        self.matrix, self.bias = rows_of(c_out, c, F32, 66, scale=c ** -0.5), rows_of(1, c_out, F32, 67)[0]
        self.offsets = torch.tensor([0, 250, 250, n], dtype=torch.int32, device="cuda")
        self.state = torch.tensor([SEED, STEP], device="cuda")

    def forward(self):
        p = self.p
        y = p.pcpp_group_norm_fwd(self.x, self.groups, self.w, self.b, self.offsets, act=p.ACT_SILU, p=0.1, random=p.Random(self.state, 1))
        h = p.pcpp_mx_pack(y.y, columns=True)
        m = p.pcpp_mx_pack(self.matrix, columns=True)
        f = p.pcpp_mx_product(h.rows, m.rows, self.bias, dtype=self.dtype)
        return y, h, m, f, p.pcpp_dropout_fwd(f, 0.2, p.Random(self.state, 2), self.residual)

    def step(self):
        p = self.p
        y, h, m, f, out = self.forward()
        df = p.pcpp_dropout_bwd(self.dy, 0.2, p.Random(self.state, 2), dtype=self.dtype)
        d = p.pcpp_mx_pack(df, columns=True, random=p.Random(self.state, 3))
        dh = p.pcpp_mx_product(d.rows, m.columns, dtype=self.dtype)
        dm = p.pcpp_mx_product(d.columns, h.columns, dtype=F32)
        g = p.pcpp_group_norm_bwd(dh, self.x, y.mean_rstd, self.w, self.b, self.offsets, act=p.ACT_SILU, p=0.1, random=p.Random(self.state, 1))
        return {"y": y.y, "f": f, "out": out, "df": df, "dh": dh, "dm": dm, "dx": g.dx, "dw": g.dw, "db": g.db}


@gpu
def test_a_layer_forward_and_back(pcpp):
    """Every stage against its 64-bit form on what the stage before it gave."""
    L = Layer(pcpp)
    o = L.step()
    offsets = L.offsets.tolist()
    f1, f2 = factors(uniform16(SEED, STEP, 1, L.n, L.c), 0.1), factors(uniform16(SEED, STEP, 2, L.n, L.c_out), 0.2)
    y, stats, off, _ = group_norm(L.x, 8, L.w, L.b, offsets, "silu", 1e-5, f1)
    within(o["y"], y, off, "norm")
    h = o["y"].double().cpu().numpy()
    m = L.matrix.double().cpu().numpy()
    values = lambda x, u=None: torch.from_numpy(to_bits(x, u)[2])  # noqa: E731
    ref, off = product_reference(values(h), values(m), L.bias.double().cpu(), "none")
    within(o["f"], ref, off, "linear")
    branch = torch.from_numpy(f2) * o["f"].double().cpu()
    within(o["out"], L.residual.double().cpu() + branch, 2 * U * (branch.abs() + L.residual.double().cpu().abs()), "out")
    within(o["df"], torch.from_numpy(f2) * L.dy.double().cpu(), U * (torch.from_numpy(f2) * L.dy.double().cpu()).abs(), "df")
    df = o["df"].double().cpu().numpy()
    u = uniform16(SEED, STEP, 3, L.n, L.c_out)
    within(o["dh"], *product_reference(values(df, u), values(m.T), None, "none"), "dh")
    within(o["dm"], *product_reference(values(df.T, u.T), values(h.T), None, "none"), "dm")
    y2 = pcpp.pcpp_group_norm_fwd(L.x, 8, L.w, L.b, L.offsets, act=pcpp.ACT_SILU, p=0.1, random=pcpp.Random(L.state, 1))
    refs = group_norm_grads(o["dh"], L.x, y2.mean_rstd, L.w, L.b, offsets, "silu", f1)
    for name, ref in zip(("dx", "dw", "db"), refs):
        within(o[name], *ref, name)


@gpu
def test_a_captured_layer_draws_anew_with_every_step(pcpp):
    """A captured step whose state goes on between replays gives what the eager step gives from that state; eager work and a second graph
    lie between."""
    L, M = Layer(pcpp), Layer(pcpp, n=300, c=91, c_out=40)
    L.step(), M.step()
    torch.cuda.synchronize()
    graphs = []
    for layer in (L, M):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer.step()
            layer.state[1] += 1
        graphs.append((g, out, layer))
    seen = []
    for replay in range(3):
        for g, out, layer in graphs:
            layer.state.copy_(torch.tensor([SEED, 1000 + replay]))
            want = {k: v.clone() for k, v in layer.step().items()}
            for v in out.values():
                v.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert int(layer.state[1]) == 1001 + replay
            for k, v in out.items():
                assert torch.equal(v, want[k]), (replay, k)
            if layer is L:
                seen.append(want["out"])
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


@gpu
def test_streams_and_the_callers_workspaces(pcpp):
    """Calls on a stream of their own, with workspaces of the caller's; the same bits each time."""
    L = Layer(pcpp, n=3000, c=256, c_out=64)
    want = {k: v.clone() for k, v in L.step().items()}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = L.step()
    torch.cuda.current_stream().wait_stream(stream)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    lib = pcpp.library()
    need = max(lib.pcpp_group_norm_workspace_bytes(3000, 256, 3, 8, b) for b in (0, 1))
    for room in (torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty(1, dtype=torch.uint8, device="cuda"),
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(need)):
        y = pcpp.pcpp_group_norm_fwd(L.x, 8, L.w, L.b, L.offsets, act=pcpp.ACT_SILU, p=0.1, random=pcpp.Random(L.state, 1), workspace=room)
        assert torch.equal(y.y, want["y"])
        d = pcpp.pcpp_group_norm_bwd(want["dh"], L.x, y.mean_rstd, L.w, L.b, L.offsets, act=pcpp.ACT_SILU, p=0.1, random=pcpp.Random(L.state, 1), workspace=room)
        assert torch.equal(d.dx, want["dx"]) and torch.equal(d.dw, want["dw"])


@gpu
def test_outputs_that_are_given_count_as_written(pcpp):
    x = rows_of(30, 64, F32)
    w = pcpp.pcpp_mx_pack(rows_of(64, 64, F32)).rows
    for call in (lambda out: pcpp.pcpp_dropout_fwd(x, 0.5, rng(pcpp), out=out), lambda out: pcpp.pcpp_dropout_bwd(x, 0.5, rng(pcpp), out=out),
                 lambda out: pcpp.pcpp_group_norm_fwd(x, 4, out=out).y, lambda out: pcpp.pcpp_mx_linear(x, w, out=out),
                 lambda out: pcpp.pcpp_mx_unpack(w, out=out[:64] if out.shape[0] >= 64 else torch.empty(64, 64, device="cuda"))):
        out = torch.empty_like(x)
        before = out._version
        y = call(out)
        assert y.data_ptr() != out.data_ptr() or out._version > before


# ---- past 32 bits ------------------------------------------------------------------------------------------------

@gpu
def test_tensors_past_four_gibibytes(pcpp):
    n, c = 2_200_000, 1024
    last = 3000
    x = torch.empty(n, c, dtype=BF16, device="cuda")
    x[:last], x[-last:] = 1.0, rows_of(last, c, BF16, 71)
    tail = x[-last:].double().cpu()
    y = pcpp.pcpp_dropout_fwd(x, 0.25, rng(pcpp))
    k = torch.from_numpy(factors(uniform16(SEED, STEP, 3, np.arange(n - 64, n), c), 0.25))
    within(y[-64:], k * tail[-64:], U * (k * tail[-64:]).abs(), "dropout")
    # one cloud, of the last rows
    off = torch.tensor([n - last, n], dtype=torch.int32, device="cuda")
    z = pcpp.pcpp_group_norm_fwd(x, 32, None, None, off, out=y, act=pcpp.ACT_SILU)
    ref, stats, off_y, off_stats = group_norm(tail.to(BF16), 32, None, None, None, "silu", 1e-5, None)
    within(z.y[-last:], ref, off_y, "norm")
    within(z.mean_rstd, stats, off_stats, "mean_rstd")
    d = pcpp.pcpp_group_norm_bwd(x, x, z.mean_rstd, None, None, off, act=pcpp.ACT_SILU)
    refs = group_norm_grads(tail.to(BF16), tail.to(BF16), z.mean_rstd, None, None, None, "silu", None)
    within(d.dx[-last:], *refs[0], "dx")
    within(d.dw, *refs[1], "dw")
    del d, y, z
    m = pcpp.pcpp_mx_pack(x, columns=True)
    assert (m.rows.q[-64:].cpu().numpy() == to_bits(tail[-64:].numpy())[0]).all()
    blocks = 128                                       # of the last rows, all channels: the columns' last blocks
    lo = n - n % 32 - 32 * blocks + 32
    lo = max(lo, n - last + (-(n - last)) % 32)
    part = to_bits(x[lo:].double().cpu().numpy().T)
    assert (m.columns.q[:, lo // 2:].cpu().numpy() == part[0]).all()
    v = pcpp.pcpp_mx_unpack(m.rows)
    assert (v[-64:].double().cpu().numpy() == to_bits(tail[-64:].numpy())[2]).all()
    del v
    w = pcpp.pcpp_mx_pack(rows_of(1024, c, F32, 72, scale=c ** -0.5)).rows
    out = pcpp.pcpp_mx_product(m.rows, w)
    ref, off_y = product_reference(torch.from_numpy(to_bits(tail[-64:].numpy())[2]), pcpp.pcpp_mx_unpack(w, F32).double().cpu(), None, "none")
    within(out[-64:], ref, off_y, "product")
