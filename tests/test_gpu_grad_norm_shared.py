"""Gradients that several tensors share, in the norm, in a scaled copy and in place."""
import numpy as np
import pytest
import torch

from tests.test_gpu_grad_norm import U, ctx, f64, gradients, plan, qrm  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [[300, 300, 7], [7, 300, 300], [5000, 3, 5000]])
def test_a_gradient_that_two_tensors_share(qrm, ctx, sizes):
    opt, grads = plan(qrm, ctx, sizes, torch.float32), gradients(sizes, torch.float32)
    twice = [i for i, n in enumerate(sizes) if sizes.count(n) == 2]
    grads[twice[1]] = grads[twice[0]]
    before = [g.clone() for g in grads]
    norm, scale = torch.empty(1, device="cuda"), torch.full((1,), 0.5, device="cuda")
    opt.qrm_adamw_grad_norm(grads, 1.0, norm, None)                            # it counts twice
    outs = [torch.empty_like(g) for g in grads]
    opt.qrm_adamw_scale_grads(grads, scale, outs)
    with pytest.raises(qrm.QrmError) as e:
        opt.qrm_adamw_scale_grads(grads, scale)
    assert e.value.status == qrm.QRM_E_INVALID and "two outputs" in e.value.message
    with pytest.raises(qrm.QrmError):
        opt.qrm_adamw_scale_grads(before, scale, [outs[twice[0]] if i in twice else o for i, o in enumerate(outs)])
    torch.cuda.synchronize()
    want = np.sqrt(sum(float((f64(g) ** 2).sum()) for g in grads))
    assert abs(float(norm) - want) <= (U + 2.0 ** -40) * want
    assert all(torch.equal(g, b) for g, b in zip(grads, before)), "a refused call has written"
    assert all(torch.equal(o, b * 0.5) for o, b in zip(outs, before))
    opt.close()


def test_outputs_in_any_order_and_empty_ones(qrm, ctx):
    """Addresses that fall, and tensors without elements at one address."""
    sizes = [100, 0, 5000, 0, 3]
    opt, grads = plan(qrm, ctx, sizes, torch.bfloat16), gradients(sizes, torch.bfloat16)
    buffer = torch.zeros(3 * 8192, dtype=torch.bfloat16, device="cuda")
    outs = [buffer[8192 * k:8192 * k + n] for k, n in zip((2, 2, 1, 2, 0), sizes)]
    opt.qrm_adamw_scale_grads(grads, torch.full((1,), 0.25, device="cuda"), outs)
    torch.cuda.synchronize()
    assert all(torch.equal(o, g * 0.25) for o, g in zip(outs, grads))
    opt.close()
