"""What the entry points of the operators around the convolution refuse, before any GPU call."""
import ctypes

import pytest

F32, BF16 = 0, 1
INVALID, WORKSPACE, UNSUPPORTED = -1, -3, -4


@pytest.fixture(scope="module")
def lib():
    from paper_2511_23227_amd import binding
    return binding.library()


@pytest.fixture(scope="module")
def p():
    """A 256-byte aligned address; nothing is read from it."""
    buf = ctypes.create_string_buffer(8192)
    at = (ctypes.addressof(buf) + 255) // 256 * 256
    p.keep = buf
    return at


def vp(at):
    return ctypes.c_void_p(at)


def test_pack(lib, p):
    a = vp(p)
    assert [lib.pcpp_act_code_bytes(c) for c in (0, 1, 128, 129, 1024, 1025)] == [0, 4, 4, 8, 32, 0]
    for fn, args in ((lib.pcpp_act_pack, lambda x, d, n, c, q, e: (x, d, n, c, q, e, None)),
                     (lib.pcpp_act_unpack, lambda x, d, n, c, q, e: (q, e, n, c, x, d, None))):
        assert fn(*args(a, F32, -1, 8, a, a)) == INVALID
        assert fn(*args(a, F32, 4, 0, a, a)) == UNSUPPORTED
        assert fn(*args(a, F32, 4, 1025, a, a)) == UNSUPPORTED
        assert fn(*args(a, F32, 2 ** 31 - 1, 8, a, a)) == UNSUPPORTED
        assert fn(*args(a, 7, 4, 8, a, a)) == UNSUPPORTED
        assert fn(*args(None, F32, 4, 8, a, a)) == INVALID
        assert fn(*args(a, F32, 4, 8, None, a)) == INVALID
        assert fn(*args(a, F32, 4, 8, a, None)) == INVALID
        assert fn(*args(vp(p + 4), F32, 4, 8, a, a)) == INVALID and b"aligned" in lib.pcpp_last_error()
        assert fn(*args(a, F32, 4, 8, a, vp(p + 1))) == INVALID
        assert fn(*args(None, F32, 0, 8, None, None)) == 0                          # no rows: nothing to do


def test_weight_gradient_from_packed_input(lib, p):
    a = vp(p)
    need = lib.pcpp_mvmr_packed_workspace_bytes(100, 100, 50, 16, 8, 27, BF16)
    assert need >= lib.pcpp_mvmr_workspace_bytes(2, 100, 100, 50, 16, 8, 27, BF16) > 0
    # the copy of x that one shape needs
    assert lib.pcpp_mvmr_packed_workspace_bytes(1000, 100, 50, 256, 256, 27, BF16) == \
        lib.pcpp_mvmr_workspace_bytes(2, 1000, 100, 50, 256, 256, 27, BF16) + 1000 * 256 * 2
    assert lib.pcpp_mvmr_packed_workspace_bytes(-1, 100, 50, 16, 8, 27, BF16) == 0

    def call(q=a, e=a, dy=a, dw=a, dtype=BF16, n_in=100, c_in=16, K=27, tri=a, plan=(None, 0, 0), ws=(a, need), n_out=100, n_tri=50, c_out=8):
        return lib.pcpp_mvmr_bwd_weight_packed(q, e, dy, dw, dtype, n_in, n_out, c_in, c_out, K, tri, tri, tri, tri, n_tri, *plan, *ws, None)

    assert call(q=None) == INVALID and call(e=None) == INVALID and call(dy=None) == INVALID and call(dw=None) == INVALID
    assert call(n_in=-1) == INVALID and call(K=26) == INVALID and call(tri=None) == INVALID
    assert call(c_in=1025) == UNSUPPORTED and call(dtype=5) == UNSUPPORTED and call(K=343) == UNSUPPORTED
    assert call(e=vp(p + 2)) == INVALID and call(q=vp(p + 8)) == INVALID
    assert call(ws=(None, need)) == WORKSPACE and call(ws=(a, need - 1)) == WORKSPACE and call(ws=(vp(p + 16), need)) == WORKSPACE
    assert call(plan=(a, 10, 1)) == WORKSPACE                                       # a plan that is given has to fit
    assert call(plan=(a, 1 << 30, 2)) == INVALID
    # tensors past 4 GiB cannot do without one
    big = dict(n_in=5_000_000, n_out=5_000_000, c_in=1000, n_tri=1000)
    need_big = lib.pcpp_mvmr_packed_workspace_bytes(5_000_000, 5_000_000, 1000, 1000, 8, 27, BF16)
    assert call(**big, ws=(a, need_big)) == INVALID and b"plan" in lib.pcpp_last_error()


def fwd(lib, a, x=..., f=..., ld_f=64, gate=None, ld_gate=64, cols=0, w=None, post=1, pre=1, scale=1.0, eps=1e-6, n=4, c=64, stream=F32, dtype=F32, r=...,
        h=..., fq=None, fe=None, hq=None, he=None):
    d = lambda v: a if v is ... else v  # noqa: E731
    return lib.pcpp_block_norm_fwd(d(x), d(f), ld_f, gate, ld_gate, cols, w, w, post, pre, scale, eps, n, c, stream, dtype, d(r), d(h), fq, fe, hq, he, None)


def test_block_norm_forward(lib, p):
    a = vp(p)
    call = lambda **k: fwd(lib, a, **k)  # noqa: E731
    assert call(n=-1) == INVALID and call(c=0) == UNSUPPORTED and call(c=1025, ld_f=1025) == UNSUPPORTED and call(n=2 ** 31) == UNSUPPORTED
    assert call(stream=BF16, dtype=F32) == UNSUPPORTED and call(dtype=9) == UNSUPPORTED
    assert call(post=3) == INVALID and call(pre=-1) == INVALID
    assert call(eps=-1.0) == INVALID and call(eps=float("nan")) == INVALID and call(scale=float("inf")) == INVALID
    assert call(cols=2) == INVALID and call(cols=64) == INVALID and call(gate=a) == INVALID and call(gate=a, cols=64, ld_gate=63) == INVALID
    assert call(ld_f=63) == INVALID and call(x=None) == INVALID and call(r=None) == INVALID and call(h=None) == INVALID
    assert call(pre=0) == INVALID                                                   # h without a norm
    assert call(f=None) == INVALID                                                  # r without a block
    assert call(f=None, r=None, pre=0, h=None) == INVALID                           # nothing to do
    assert call(f=None, r=None, gate=a, cols=64) == INVALID and call(f=None, r=None, fq=a, fe=a) == INVALID
    assert call(fq=a) == INVALID and call(he=a) == INVALID and call(pre=0, h=None, hq=a, he=a) == INVALID
    assert call(x=vp(p + 8)) == INVALID and call(f=vp(p + 2)) == INVALID and call(w=vp(p + 2)) == INVALID and call(fq=vp(p + 8), fe=a) == INVALID
    assert call(n=0, x=None, f=None, r=None, h=None) == 0


def test_block_norm_backward(lib, p):
    a = vp(p)
    need = lib.pcpp_block_norm_workspace_bytes(4, 64)
    assert need > 0 and lib.pcpp_block_norm_workspace_bytes(-1, 64) == 0 and lib.pcpp_block_norm_workspace_bytes(4, 1025) == 0

    def call(dr=a, dh=a, r=a, f=a, ld_f=64, fq=None, fe=None, gate=None, ld_gate=64, cols=0, w=None, post=1, pre=1, scale=1.0, eps=1e-6, n=4, c=64,
             stream=F32, dtype=F32, dx=a, df=a, dgate=None, dwp=a, dwn=a, ws=(a, need)):
        return lib.pcpp_block_norm_bwd(dr, dh, r, f, ld_f, fq, fe, gate, ld_gate, cols, w, w, post, pre, scale, eps, n, c, stream, dtype, dx, df, dgate,
                                       dwp, dwn, *ws, None)

    assert call(n=-1) == INVALID and call(c=1025, ld_f=1025) == UNSUPPORTED and call(stream=BF16) == UNSUPPORTED
    assert call(dh=None) == INVALID and call(r=None) == INVALID and call(pre=0) == INVALID
    assert call(dr=None, dh=None, r=None, pre=0, dwn=None) == INVALID               # nothing flows
    assert call(fq=a, fe=a) == INVALID and call(f=None, fq=a) == INVALID and call(f=None) == INVALID
    assert call(df=None) == INVALID and call(dgate=a) == INVALID and call(gate=a, cols=64) == INVALID
    assert call(f=None, post=0) == INVALID and call(pre=0, dh=None, r=None) == INVALID      # a weight's gradient without f, or without its norm
    assert call(dx=vp(p + 8)) == INVALID and call(dwp=vp(p + 2)) == INVALID
    assert call(ws=(None, need)) == WORKSPACE and call(ws=(a, need - 1)) == WORKSPACE and call(ws=(vp(p + 64), need)) == WORKSPACE


def test_log_probs(lib, p):
    a = vp(p)

    def call(x=a, dtype=F32, n=4, v=100, ld=100, labels=a, top=2, tv=a, ti=a, ws=(None, 0), lse=a):
        return lib.pcpp_log_probs_fwd(x, dtype, n, v, ld, labels, top, a, a, lse, tv, ti, *ws, None)

    assert call(n=-1) == INVALID and call(v=0) == INVALID and call(ld=99) == INVALID and call(dtype=2) == UNSUPPORTED
    assert call(n=2 ** 31) == UNSUPPORTED and call(v=2 ** 31, ld=2 ** 31) == UNSUPPORTED
    assert call(x=None) == INVALID and call(x=vp(p + 2)) == INVALID and call(labels=vp(p + 2)) == INVALID and call(lse=vp(p + 1)) == INVALID
    assert call(top=-1) == INVALID and call(top=65) == INVALID and call(v=2, ld=2, top=3) == INVALID
    assert call(tv=None) == INVALID and call(ti=None) == INVALID
    need = lib.pcpp_log_probs_workspace_bytes(1, 200_000, 20)
    assert need > 0 and lib.pcpp_log_probs_workspace_bytes(4, 100, 2) == 0 and lib.pcpp_log_probs_workspace_bytes(1, 200_000, 65) == 0
    big = dict(n=1, v=200_000, ld=200_000, top=20)
    assert call(**big) == WORKSPACE and call(**big, ws=(a, need - 1)) == WORKSPACE and call(**big, ws=(vp(p + 8), need)) == WORKSPACE
    assert call(n=0, x=None) == 0

    def back(x=a, dtype=F32, n=4, v=100, ld=100, lse=a, entropy=a, dl=a, dh=a, out=vp(p + 16), ld_d=100):
        return lib.pcpp_log_probs_bwd(x, dtype, n, v, ld, a, lse, entropy, dl, dh, out, ld_d, None)

    assert back(n=-1) == INVALID and back(ld_d=99) == INVALID and back(lse=None) == INVALID and back(out=None) == INVALID
    assert back(entropy=None) == INVALID and back(out=vp(p + 2)) == INVALID and back(dtype=4) == UNSUPPORTED
    assert back(out=a, ld_d=104) == INVALID                                         # in place with another pitch
    assert back(n=0, x=None) == 0
