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
