"""pack_codes: the type that the packed codes come in is that of the projections that read them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_types_of_packed_codes():
    from paper_2601_11546_amd import binding as rs
    w = torch.randint(0, 256, (260, 128), dtype=torch.uint8, device="cuda")
    packed = rs.pack_codes(w)
    torch.cuda.synchronize()
    assert packed.dtype is torch.uint8 and torch.equal(packed.view(2, 1, 256, 128)[0, 0], w[:256]) and torch.equal(packed.view(2, 1, 256, 128)[1, 0, :4], w[256:])
    for dtype, want in ((torch.int8, torch.int8), (torch.float8_e4m3fn, torch.uint8)):
        again = rs.pack_codes(w.view(dtype))
        torch.cuda.synchronize()
        assert again.dtype is want and torch.equal(again.view(torch.uint8), packed)
