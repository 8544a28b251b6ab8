"""The operators around the convolution where sizes, storage and the caller's own tensors are out of the ordinary."""
import io

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def pcpp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_23227_amd as m
    m.library()
    return m


def test_packed_weight_gradient_whose_codes_pass_32_bit_offsets(pcpp):
    """2^30 rows of one channel: 1 GiB of q, 4 GiB of codes.  Integers below 128 times powers of two are exact in 8 bits, in the products and in their
    sums, and rows far apart have different codes."""
    if torch.cuda.get_device_properties(0).total_memory < 64 << 30:
        pytest.skip("needs 64 GiB")
    n_in, n_out, c_out = 2 ** 30 + 9, 40, 3
    at = torch.tensor([0, 1, 2 ** 20, 2 ** 29, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, n_in - 1], device="cuda")
    value = torch.tensor([127.0, -64.0, 96.0, 100.0, -80.0, 65.0, -127.0, 72.0], device="cuda") * 2.0 ** torch.arange(-4.0, 4.0, device="cuda")
    p = pcpp.Packed(torch.zeros(n_in, 1, dtype=torch.int8, device="cuda"), torch.ones(n_in, 4, dtype=torch.uint8, device="cuda"))
    few = pcpp.pcpp_act_pack(value[:, None].contiguous())
    p.q[at], p.codes[at] = few.q, few.codes
    dy = torch.arange(n_out * c_out, device="cuda").view(n_out, c_out).to(BF16)
    o = torch.tensor([0, 3, 39, 7, 7, 8, 20, 21], dtype=torch.int32, device="cuda")
    cell = torch.tensor([0, 0, 0, 2, 2, 2, 5, 7], dtype=torch.int32, device="cuda")
    seg = torch.searchsorted(cell, torch.arange(9, dtype=torch.int32, device="cuda"))
    T = pcpp.Triplets(o, at.int(), cell, seg, 8, n_in, n_out, 2, None, 0)
    ref = torch.zeros(8, c_out, 1, dtype=torch.float64, device="cuda")
    ref.index_add_(0, cell.long(), (dy[o.long()].double() * value[:, None].double())[..., None])
    assert torch.equal(pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, T).double(), ref)


def expanded(n):
    """One byte that says it is n: what is written past it belongs to others."""
    return torch.full((1,), 7, dtype=torch.uint8, device="cuda").expand(max(int(n), 1))


def test_workspaces_that_do_not_lie_in_one_piece(pcpp):
    """A caller's workspace of enough bytes is used only if they are there: an expanded one is left alone, and the results are the same."""
    g = torch.Generator(device="cuda").manual_seed(3)
    lib = pcpp.library()
    n, c = 900, 48
    x, dy = (torch.randn(n, c, generator=g, device="cuda").to(BF16) for _ in range(2))
    xyz = torch.rand(n, 3, generator=g, device="cuda")
    T = pcpp.pcpp_build_triplets(xyz, xyz, 0.15, 3)
    p = pcpp.pcpp_act_pack(x)
    w = torch.randn(T.K, c, c, generator=g, device="cuda").to(BF16)
    sizes = (n, n, T.n_triplets, c, c, T.K, 1)
    logits = torch.randn(2, 20_000, generator=g, device="cuda")

    def fields(y):
        return [t for t in vars(y).values() if t is not None] if hasattr(y, "__dict__") else [y.log_prob, y.entropy, y.top_log_prob, y.top_index]

    labels = torch.zeros(2, dtype=torch.int32, device="cuda")
    for need, call in (
            (lib.pcpp_mvmr_packed_workspace_bytes(*sizes), lambda **k: [pcpp.pcpp_mvmr_bwd_weight_packed(p, dy, T, **k)]),
            (lib.pcpp_block_norm_workspace_bytes(n, c), lambda **k: fields(pcpp.pcpp_block_norm_bwd(dy, dy, x, x, **k))),
            (lib.pcpp_log_probs_workspace_bytes(2, 20_000, 5), lambda **k: fields(pcpp.pcpp_log_probs_fwd(logits, labels, 5, **k))),
            (lib.pcpp_mvmr_workspace_bytes(0, *sizes), lambda **k: [pcpp.pcpp_mvmr_fwd(x, w, T, **k)]),
            (lib.pcpp_mvmr_workspace_bytes(1, *sizes), lambda **k: [pcpp.pcpp_mvmr_bwd_input(dy, w, T, **k)]),
            (lib.pcpp_mvmr_workspace_bytes(2, *sizes), lambda **k: [pcpp.pcpp_mvmr_bwd_weight(x, dy, T, **k)])):
        assert need > 512
        space = expanded(need)
        for a, b in zip(call(), call(workspace=space)):
            assert torch.equal(a, b)
        assert int(space[0]) == 7
        whole = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
        for a, b in zip(call(), call(workspace=whole)):
            assert torch.equal(a, b)
        assert (whole != 7).any()                      # (one piece: it is used)


def test_triplets_into_buffers_that_do_not_lie_in_one_piece(pcpp):
    g = torch.Generator(device="cuda").manual_seed(4)
    xyz = torch.rand(700, 3, generator=g, device="cuda")
    ref = pcpp.pcpp_build_triplets(xyz, xyz, 0.15, 3)
    one = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    space = expanded(1 << 28)
    T = pcpp.pcpp_build_triplets(xyz, xyz, 0.15, 3, buffers={"workspace": space, "plan": space, "tri_o": one.expand(1 << 20)})
    assert torch.equal(T.tri_o, ref.tri_o) and torch.equal(T.tri_i, ref.tri_i) and torch.equal(T.tri_k, ref.tri_k)
    assert pcpp.pcpp_count_triplets(xyz, xyz, 0.15, 3, workspace=space) == ref.n_triplets
    assert int(space[0]) == 7 and int(one[0]) == 7


def test_outputs_have_storages_of_their_own(pcpp):
    """What a call returns can be saved, alone and together, holds no more memory than its own, and can be resized without reaching another."""
    g = torch.Generator(device="cuda").manual_seed(5)
    n, c = 70, 40
    x, f, gate, dr = (torch.randn(n, c, generator=g, device="cuda") for _ in range(4))
    w = torch.ones(c, device="cuda")
    y = pcpp.pcpp_block_norm_fwd(x, f, gate, w, w, pack_f=True, pack_h=True)
    b = pcpp.pcpp_block_norm_bwd(dr, dr, y.r, f, gate, w, w)
    p = pcpp.pcpp_act_pack(x)
    lp = pcpp.pcpp_log_probs_fwd(x, torch.zeros(n, dtype=torch.int32, device="cuda"), 5)
    split = pcpp.pcpp_log_probs_fwd(x.view(1, -1).repeat(1, 5), torch.zeros(1, dtype=torch.int32, device="cuda"), 5)
    results = dict(r=y.r, h=y.h, fq=y.f_packed.q, fcodes=y.f_packed.codes, hq=y.h_packed.q, hcodes=y.h_packed.codes, dx=b.dx, df=b.df, dgate=b.dgate,
                   dw_post=b.dw_post, dw_pre=b.dw_pre, q=p.q, codes=p.codes)
    for name, l in (("lp", lp), ("split", split)):
        results.update({name + k: getattr(l, k) for k in ("log_prob", "entropy", "max_log_sum", "top_log_prob", "top_index")})
    at = [t.untyped_storage().data_ptr() for t in results.values()]
    assert len(set(at)) == len(at)
    for name, t in results.items():
        assert t.storage_offset() == 0 and t.untyped_storage().nbytes() == t.numel() * t.element_size(), name
    file = io.BytesIO()
    torch.save(results, file)
    file.seek(0)
    for name, t in torch.load(file, weights_only=True).items():
        assert torch.equal(t, results[name]), name


def test_outputs_that_the_caller_gives_are_seen_by_autograd(pcpp):
    """A call that writes a caller's tensor raises its version, so that a graph that saved the tensor refuses to use what now stands there."""
    g = torch.Generator(device="cuda").manual_seed(6)
    n, c = 60, 32
    labels = torch.arange(n, dtype=torch.int32, device="cuda") % c
    head = torch.randn(c, c, generator=g, device="cuda", requires_grad=True)
    logits = torch.randn(n, c, generator=g, device="cuda") @ head
    penalty = (logits * logits).sum()                  # (saves the logits)
    y = pcpp.pcpp_log_probs_fwd(logits, labels)
    pcpp.pcpp_log_probs_bwd(logits, labels, y, torch.ones(n, device="cuda"), out=logits)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        penalty.backward()

    x = torch.randn(n, c, generator=g, device="cuda")
    xyz = torch.rand(n, 3, generator=g, device="cuda")
    T = pcpp.pcpp_build_triplets(xyz, xyz, 0.4, 2)
    w = torch.randn(T.K, c, c, generator=g, device="cuda")
    p, rows = pcpp.pcpp_act_pack(x), torch.empty(n, c, device="cuda")
    dw = torch.empty(T.K, c, c, device="cuda")
    kept = pcpp.Packed(torch.empty_like(p.q), torch.empty_like(p.codes))
    buffers = {k: torch.empty(48 * 1024, dtype=torch.int32, device="cuda") for k in ("tri_o", "tri_i", "tri_k")}
    for call, given in ((lambda: pcpp.pcpp_act_pack(x, out=kept), (kept.q, kept.codes)),
                        (lambda: pcpp.pcpp_act_unpack(p, out=rows), (rows,)),
                        (lambda: pcpp.pcpp_mvmr_bwd_weight_packed(p, x, T, dw=dw), (dw,)),
                        (lambda: pcpp.pcpp_mvmr_fwd(x, w, T, out=rows), (rows,)),
                        (lambda: pcpp.pcpp_mvmr_fwd_static(x, w, T, rows), (rows,)),
                        (lambda: pcpp.pcpp_mvmr_bwd_input(x, w, T, dx=rows), (rows,)),
                        (lambda: pcpp.pcpp_mvmr_bwd_weight(x, x, T, dw=dw), (dw,)),
                        (lambda: pcpp.pcpp_build_triplets(xyz, xyz, 0.4, 2, buffers=buffers), tuple(buffers.values()))):
        before = [t._version for t in given]
        call()
        assert all(t._version > v for t, v in zip(given, before))
    with torch.inference_mode():                       # (such tensors have no version)
        inference = torch.empty(n, c, device="cuda")
    assert torch.equal(pcpp.pcpp_act_unpack(p, out=inference), pcpp.pcpp_act_unpack(p, F32))
    assert torch.equal(pcpp.pcpp_mvmr_fwd(x, w, T, out=inference), pcpp.pcpp_mvmr_fwd(x, w, T))


@pytest.mark.parametrize("c", [1, 7, 20, 32, 91, 128, 640])
def test_pack_of_the_largest_numbers(pcpp, c):
    """Finite magnitudes from 127.5 steps of 2^121 on, the type's largest and lowest among them, stay at 127 steps: the next power of two would round them to
    2^128.  Others of their block are rounded in the same steps, and Inf is still Inf's code."""
    step = 2.0 ** 121
    for dtype in (F32, BF16):
        top = torch.finfo(dtype)
        x = torch.zeros(8, c, dtype=torch.float64)
        x[0], x[1], x[2], x[3] = top.max, top.min, 127.25 * step, -127.5 * step
        x[4, ::2], x[4, 1::2] = top.max, 3.5 * step
        x[5], x[6] = 63.75 * step, 100 * step
        x[6, -1] = top.min
        x = x.to(dtype).cuda()
        p = pcpp.pcpp_act_pack(x)
        blocks = -(-c // 32)
        assert (p.codes[:7, :blocks] == 248).all() and (p.codes[7, :blocks] == 1).all()
        steps = (x.double() / step).round().clamp(-127, 127)
        assert torch.equal(p.q.double(), steps)
        for out in (F32, BF16):
            assert torch.equal(pcpp.pcpp_act_unpack(p, out).double(), steps * step)
        x[0, 0] = float("inf")
        assert int(pcpp.pcpp_act_pack(x).codes[0, 0]) == 255
        y = pcpp.pcpp_block_norm_fwd(torch.zeros(1, c, device="cuda"), x[1:2], None, post_norm=0, pack_f=True)
        assert torch.equal(y.f_packed.q, p.q[1:2]) and torch.equal(y.f_packed.codes, p.codes[1:2])


@pytest.mark.parametrize("kind", [1, 2])
def test_block_norm_of_rows_past_the_range_of_squares(pcpp, kind):
    """Finite rows whose sum of squares is past fp32 come out as zero, not as NaN, and reach no other row; just under the line they are normal."""
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(5, 64, generator=g, device="cuda")
    ref = pcpp.pcpp_block_norm_fwd(x, None, pre_norm=kind).h
    big = x.clone()
    big[1] *= 2.0 ** 70
    big[3] *= 2.0 ** 55                                # (eps is nothing beside either)
    h = pcpp.pcpp_block_norm_fwd(big, None, pre_norm=kind).h
    assert not h[1].any() and torch.equal(h[[0, 2, 4]], ref[[0, 2, 4]]) and torch.allclose(h[3], ref[3], rtol=0, atol=1e-5)
    ones = torch.ones_like(x)
    d = pcpp.pcpp_block_norm_bwd(None, ones, big, pre_norm=kind)
    assert not d.dx[1].any() and torch.isfinite(d.dx).all() and torch.isfinite(d.dw_pre).all()
