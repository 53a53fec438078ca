"""The fine-tuning example's autograd functions without a GPU: the library's calls are stood in for."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import finetune_decoder
    finally:
        sys.path.pop(0)
    return finetune_decoder


class Calls:
    """y = x^2, loss = sum of squares of the logits."""

    def qrm_group_norm(self, desc, x, gamma, beta, y, mean, rstd):
        y.copy_(x.detach().square())

    def qrm_group_norm_backward(self, desc, x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta):
        dx.copy_(2.0 * x.detach() * dy.detach())
        dgamma.zero_(), dbeta.zero_()

    def qrm_message_loss(self, logits, target, rows, n, bits, weight, loss, grad, errors):
        loss.copy_(logits.detach().square().sum().view(1))
        grad.copy_(2.0 * logits.detach())


def test_first_derivatives_go_through_and_second_ones_are_refused(example):
    """The functions know their first derivative alone: a second one must not come out without their share."""
    x = torch.randn((2, 3, 3, 4), requires_grad=True)
    gamma, beta = torch.ones(4, requires_grad=True), torch.zeros(4, requires_grad=True)
    logits = torch.randn((2, example.BITS), requires_grad=True)
    for value, of in ((example.NormAct.apply(x, gamma, beta, Calls(), 2).sum(), x), (example.MessageLoss.apply(logits, None, Calls(), 1.0, None), logits)):
        first, = torch.autograd.grad(value, of, create_graph=True)
        assert torch.allclose(first, 2.0 * of)
        with pytest.raises(RuntimeError, match="differentiated again"):
            torch.autograd.grad(first.square().sum() + of.square().sum(), of)
        first, = torch.autograd.grad((example.NormAct.apply(x, gamma, beta, Calls(), 2).sum() if of is x else example.MessageLoss.apply(logits, None, Calls(), 1.0, None)), of)
        assert torch.allclose(first, 2.0 * of) and not first.requires_grad
