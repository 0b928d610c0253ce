"""oscar_verify_drafts of a step without drafts, whose tensors may then be left out."""
import pytest

pytestmark = pytest.mark.gpu


def test_no_drafts_at_all():
    import torch
    from paper_2605_19660_amd import binding as ob
    g = torch.Generator().manual_seed(1)
    p, u = torch.rand(3, 1, 5003, generator=g).cuda(), torch.rand(3, 1, generator=g).cuda()
    want = ob.verify_drafts(p, p[:, :0].contiguous(), torch.empty(3, 0, dtype=torch.int32, device="cuda"), u)
    got = ob.verify_drafts(p, None, None, u)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[0].tolist() == [1, 1, 1]
    with pytest.raises(AssertionError):
        ob.verify_drafts(torch.rand(3, 2, 10, device="cuda"), None, None, torch.rand(3, 2, device="cuda"))
