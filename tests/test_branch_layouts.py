"""Matrices in 8 bits whose tensors were changed in place after a call had found them in order: the C side gets addresses alone, so the
binding has to refuse them in every call, whatever an earlier one found."""
import pytest
import torch

from paper_2603_06626_b200 import binding as B


def _resized(q):
    q.codes.resize_(32, 16)


def _turned(q):
    q.codes.t_()              # square: the same shape, other strides


def _swapped(q):
    q.scales.data = torch.zeros(1, 1, 32, 4, 2, dtype=torch.uint8)


def _strided(q):
    q.codes.set_(torch.empty(32, 64, dtype=torch.float8_e4m3fn)[:, :32])


def _flat(q):
    q.scales.resize_(512)


CHANGES = [_resized, _turned, _swapped, _strided, _flat]


@pytest.mark.parametrize("change", CHANGES)
def test_a_matrix_that_was_changed_in_place_is_refused(change):
    q, on = B.Fp8Blocks.empty(32, 32, "cpu"), torch.device("cpu")
    B._expect_fp8("q", q, 32, 32, on)
    change(q)
    with pytest.raises((ValueError, TypeError)):
        B._expect_fp8("q", q, 32, 32, on)


@pytest.mark.parametrize("change", CHANGES)
def test_every_operand_of_every_call_is_looked_at(change):
    """On CPU tensors a call whose operands are in order ends at the check of the device; one with a changed operand ends before."""
    bf = torch.bfloat16
    x = torch.zeros(32, 32, dtype=bf)
    calls = [(lambda a, b, c: B.linear_fp8(a, b), 2), (lambda a, b, c: B.linear_fp8(b, a), 2), (lambda a, b, c: B.linear_fp8(x, a), 1),
             (lambda a, b, c: B.linear_fp8_backward(x, a, b), 2), (lambda a, b, c: B.gated_ffn_fp8(x, a, b, c), 3),
             (lambda a, b, c: B.gated_ffn_fp8(a, b, b, c), 3), (lambda a, b, c: B.dequantize_fp8(a), 1)]
    for call, used in calls:
        for which in range(used):
            q = [B.Fp8Blocks.empty(32, 32, "cpu") for _ in range(3)]
            with pytest.raises(ValueError, match="a CUDA tensor is expected"):
                call(*q)
            change(q[which])
            with pytest.raises((ValueError, TypeError)) as found:
                call(*q)
            assert "a CUDA tensor is expected" not in str(found.value)


def test_the_tensors_that_were_looked_at_are_the_ones_read():
    """A part that is set between the check and the launch (another thread's doing) does not reach the call that is under way."""
    q, on = B.Fp8Blocks.empty(32, 32, "cpu"), torch.device("cpu")
    codes, scales = q.codes, q.scales
    seen = B._expect_fp8("q", q, 32, 32, on)
    q.codes, q.scales = codes[:2], scales[..., :2]
    assert seen[0] is codes and seen[1] is scales
    with pytest.raises(ValueError):
        B._expect_fp8("q", q, 32, 32, on)
