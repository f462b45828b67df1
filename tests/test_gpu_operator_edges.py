"""Edges of the operators around the expert layer: scores that are not numbers, errors that belong to somebody else."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [8, 60, 333])
@pytest.mark.parametrize("ty", [torch.float32, torch.bfloat16])
def test_a_row_without_a_number_spoils_both_losses(E, ty):
    """Scores that are NaN throughout, or NaN beside -inf, are no empty row: the z loss is NaN as well, also where it counts alone."""
    from paper_2603_06626_b200 import binding as B
    for others in (float("nan"), -float("inf")):
        s = torch.randn(50, E, device="cuda:0").to(ty)
        s[17] = others
        s[17, E - 1] = float("nan")
        i = torch.zeros(50, 1, dtype=torch.int32, device="cuda:0")
        counts, n = B.expert_counts(i, E)
        loss, d = B.balance_loss(s, i, counts, n, balance_coef=0.0, z_coef=0.1)
        assert torch.isnan(loss).all() and torch.isnan(d[17, E - 1])
        rows = torch.arange(50, device="cuda:0") != 17
        assert torch.isfinite(d[rows]).all()
        mask = rows.to(torch.uint8)
        counts, n = B.expert_counts(i, E, mask=mask)
        loss, d = B.balance_loss(s, i, counts, n, mask=mask, balance_coef=0.0, z_coef=0.1)
        assert torch.isfinite(loss).all() and torch.isfinite(d).all()


def test_the_block_keeps_its_errors_to_itself():
    """An error of a call elsewhere is neither raised nor cleared by the block's check, and the other way round."""
    from paper_2603_06626_b200 import binding as B
    from paper_2603_06626_b200.block import RoutedBlock
    block = RoutedBlock(64, 64, 64, 8, 2, 64)
    x = torch.randn(64, 64, device="cuda:0").bfloat16()
    block.forward(x)
    block.backward(x)
    B.check_status()
    B.expert_counts(torch.full((4, 2), 9, dtype=torch.uint8, device="cuda:0"), 8)
    block.check_status()
    with pytest.raises(B.GrouterError):
        B.check_status()
    block.forward(x)
    block.status.fill_(2)
    B.check_status()
    with pytest.raises(B.GrouterError):
        block.check_status()
    block.check_status()


@pytest.mark.parametrize("E", [256, 257, 1024])
def test_losses_without_ids(E):
    from paper_2603_06626_b200 import binding as B
    s = torch.randn(40, E, device="cuda:0")
    i = s.topk(2, dim=1).indices.to(torch.int32)
    counts, n = B.expert_counts(i, E)
    want = B.balance_loss(s, i, counts, n, z_coef=0.1)
    got = B.balance_loss(s, None, counts, n, z_coef=0.1)
    B.check_status()
    assert torch.allclose(got[0], want[0], rtol=1e-5) and torch.allclose(got[1], want[1], rtol=1e-4, atol=1e-9)
