"""Four bits at the edges: forms of the product that a cost decides between, operands that lie otherwise than usual, and numbers that are not finite."""
import pytest

from test_fp4 import _linear, _matrix


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K", [(1, 640, 8192), (2, 5709, 7488), (5, 300, 2560), (7, 1000, 2560), (33, 640, 8192), (134, 156, 3520)])
def test_parts_of_few_tokens(T, O, K):
    """K shared out among CTAs, each of which has one token of its last four or fewer: every part that is read is one of a token"""
    _linear(T, O, K, 16, "bfloat16", bias=True, residual=True, seed=T + O)


@pytest.mark.gpu
def test_parts_of_few_tokens_in_a_row():
    """the same without a wait between: CTAs that have left are followed by others in their shared memory"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    ops = [(_matrix(T, K, 16, 1)[0], _matrix(O, K, 16, 2)[0], torch.empty(T, O, device="cuda"))
           for T, O, K in ((1, 640, 8192), (64, 2560, 2560), (5, 300, 2560), (134, 156, 3520), (2, 5709, 7488))]
    want = []
    for x, w, out in ops:
        bd.ssdi8_fp4_linear(x, w, out)
        torch.cuda.synchronize()
        want.append(out.clone())
    for _ in range(50):
        for x, w, out in ops:
            bd.ssdi8_fp4_linear(x, w, out)
    torch.cuda.synchronize()
    for (x, w, out), y in zip(ops, want):
        assert torch.equal(out, y)
