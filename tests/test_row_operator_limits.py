"""Sizes at which the operators around the convolution change their form, asked of the host side of the library alone."""
import pytest

F32, BF16 = 0, 1
LARGEST = 0xfffff000                                   # bytes that a kernel reaches with 32-bit offsets


@pytest.fixture(scope="module")
def lib():
    from paper_2511_23227_amd import binding
    return binding.library()


@pytest.mark.parametrize("n_in", [2 ** 30, 2 ** 30 + 7, 2 ** 31 - 2])
def test_packed_weight_gradient_whose_codes_pass_32_bit_offsets(lib, n_in):
    """A row of one channel has one byte of q and four of codes.  Where the codes take 4 GiB the kernel that reads rows in 8 bits cannot look
    them up, so the call goes by way of a bf16 copy of x, for which the workspace has room."""
    sizes = (n_in, 100, 50, 1, 8, 27, BF16)
    copy = (2 * n_in + 255) // 256 * 256
    assert lib.pcpp_mvmr_packed_workspace_bytes(*sizes) == lib.pcpp_mvmr_workspace_bytes(2, *sizes) + copy


def test_packed_weight_gradient_whose_codes_just_fit(lib):
    most = LARGEST // 4
    for n_in, copied in ((most, False), (most + 1, True)):
        sizes = (n_in, 100, 50, 1, 8, 27, BF16)
        assert (lib.pcpp_mvmr_packed_workspace_bytes(*sizes) > lib.pcpp_mvmr_workspace_bytes(2, *sizes)) == copied
    # two channels and more: x in dy's type is at least as large as the codes
    sizes = (2 ** 30 - 1024, 100, 50, 2, 8, 27, BF16)
    assert lib.pcpp_mvmr_packed_workspace_bytes(*sizes) == lib.pcpp_mvmr_workspace_bytes(2, *sizes)


@pytest.mark.parametrize("n_in,n_out,n_tri,c_in,c_out,dtype,needed", [
    (LARGEST // 4 // 64, 100, 50, 64, 8, F32, False), (LARGEST // 4 // 64 + 1, 100, 50, 64, 8, F32, True),          # x in dy's type: xq at 1 GiB
    (LARGEST // 2 // 64, 100, 50, 64, 8, BF16, False), (LARGEST // 2 // 64 + 1, 100, 50, 64, 8, BF16, True),        # ... and at 2 GiB
    (100, LARGEST // 4 // 64, 50, 8, 64, F32, False), (100, LARGEST // 4 // 64 + 1, 50, 8, 64, F32, True),          # dy
    (100, 100, LARGEST // 4, 8, 8, BF16, False), (100, 100, LARGEST // 4 + 1, 8, 8, BF16, True),                    # the list
    (2 ** 30, 100, 50, 1, 8, BF16, False),                                                                          # the codes: a copy, no plan
    (2 ** 25, 100, 50, 256, 256, BF16, False), (2 ** 25, 100, 0, 256, 8, BF16, False),                              # its own kernel; nothing to do
])
def test_packed_weight_gradient_needs_a_plan(lib, n_in, n_out, n_tri, c_in, c_out, dtype, needed):
    """The sizes from which the header asks for a plan.  (Without one the call ends there, otherwise at the workspace that is not given.)"""
    import ctypes
    buf = ctypes.create_string_buffer(512)
    a = ctypes.c_void_p((ctypes.addressof(buf) + 255) // 256 * 256)
    rc = lib.pcpp_mvmr_bwd_weight_packed(a, a, a, a, dtype, n_in, n_out, c_in, c_out, 27, a, a, a, a, n_tri, None, 0, 0, None, 0, None)
    assert (rc, b"plan is NULL" in lib.pcpp_last_error()) == ((-1, True) if needed else (-3, False))
