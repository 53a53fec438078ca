"""The example's options do what they say: --clip bounds what the optimiser takes, --attention puts the block between the decoder's others, and nothing of either runs without."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import finetune_decoder
    finally:
        sys.path.pop(0)
    return finetune_decoder


@pytest.fixture
def calls(example, monkeypatch):
    """What the example asks of the library, call by call."""
    seen = dict(norm=[], step=[], forward=0, backward=0)
    binding = example.qrm.binding
    norm, step = binding.AdamW.qrm_adamw_grad_norm, binding.AdamW.qrm_adamw_step
    forward, backward = binding.Context.qrm_attention, binding.Context.qrm_attention_backward

    def grad_norm(self, grads, max_norm, d_norm, d_scale, *args, **kw):
        norm(self, grads, max_norm, d_norm, d_scale, *args, **kw)
        size = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in grads]))
        seen["norm"].append((max_norm, float(size), d_norm.clone(), d_scale.clone(), d_scale))

    def adamw_step(self, grads, *args, d_grad_scale=None, **kw):
        seen["step"].append((len(grads), d_grad_scale, None if d_grad_scale is None else d_grad_scale.clone()))
        step(self, grads, *args, d_grad_scale=d_grad_scale, **kw)

    def attend(self, desc, *args):
        seen["forward"] += 1
        assert (desc.Lq, desc.Lk, desc.heads, desc.kv_heads, desc.D) == (256, 256, 4, 4, 16)
        forward(self, desc, *args)

    def attend_backward(self, *args):
        seen["backward"] += 1
        backward(self, *args)

    monkeypatch.setattr(binding.AdamW, "qrm_adamw_grad_norm", grad_norm)
    monkeypatch.setattr(binding.AdamW, "qrm_adamw_step", adamw_step)
    monkeypatch.setattr(binding.Context, "qrm_attention", attend)
    monkeypatch.setattr(binding.Context, "qrm_attention_backward", attend_backward)
    return seen


@pytest.mark.parametrize("clip", [0.0, 0.05])
def test_clipping(example, calls, clip):
    example.main(steps=3, attention=False, clip=clip, report=lambda s: None)
    assert len(calls["step"]) == 3 and calls["forward"] == calls["backward"] == 0
    if not clip:
        assert not calls["norm"] and all(s[1] is None for s in calls["step"])
        return
    assert len(calls["norm"]) == 3
    for (bound, size, norm, scale, where), (_, taken, value) in zip(calls["norm"], calls["step"]):
        assert bound == clip and taken is where and torch.equal(value, scale)
        assert abs(float(norm) / size - 1.0) <= 2.0 ** -20 and size > clip
        assert abs(float(scale) * size / clip - 1.0) <= 2.0 ** -20


def test_attention(example, calls):
    example.main(steps=2, attention=True, clip=0.0, report=lambda s: None)
    with_it = calls["step"][-1][0]
    assert calls["backward"] == 2 and calls["forward"] > 2
    example.main(steps=1, attention=False, clip=0.0, report=lambda s: None)
    assert calls["backward"] == 2 and calls["step"][-1][0] == with_it - 4


def test_the_blocks_parameters_are_taught(example):
    """All four of the block's have gradients that are not zero, and the images depend on it."""
    ctx = example.qrm.Context(rs=example.CODE)
    decoder = example.Decoder(torch.Generator("cuda").manual_seed(0), True)
    z = torch.randn((2, 16, 16, 8), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    images = decoder(z, ctx)
    grads = torch.autograd.grad((images * torch.randn(images.shape, generator=torch.Generator("cuda").manual_seed(2), device="cuda")).sum(), decoder.look)
    assert all(float(g.abs().max()) > 0 for g in grads)
    plain, decoder.look = decoder.look, None
    assert not torch.equal(decoder(z, ctx).detach(), images.detach())
    assert len(plain) == 4
    ctx.close()
