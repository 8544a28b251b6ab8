"""The operators around the convolution where sizes, storage and the caller's own tensors are out of the ordinary."""
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
