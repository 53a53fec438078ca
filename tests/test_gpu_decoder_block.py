"""The fine-tuning operators together, as a decoder's training step uses them: group norm, attention, message loss, clipping, AdamW."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import finetune_decoder
    finally:
        sys.path.pop(0)
    return finetune_decoder


@pytest.fixture(scope="module")
def ctx(example):
    c = example.qrm.Context(rs=example.CODE)
    yield c
    c.close()


def plain_block(x, gamma, beta, into, out, groups, heads):
    """The same block in 64 bits, differentiated by torch on the CPU."""
    n, h, w, c = x.shape
    xg = x.reshape(n, h * w, groups, c // groups)
    mean = xg.mean(dim=(1, 3), keepdim=True)
    z = ((xg - mean) / ((xg - mean).square().mean(dim=(1, 3), keepdim=True) + 1e-6).sqrt()).reshape(n, h * w, c) * gamma + beta
    q, k, v = ((z * torch.sigmoid(z)) @ into).view(n, h * w, 3, heads, -1).unbind(2)
    s = torch.einsum("nihd,njhd->nhij", q, k) * q.shape[3] ** -0.5
    o = torch.einsum("nhij,njhd->nihd", torch.softmax(s, dim=3), v).reshape(n, h * w, -1)
    return x + (o @ out).view(n, h, w, c)


def test_a_block_and_its_gradients(example, ctx):
    gen = torch.Generator().manual_seed(0)
    n, h, w, c, groups, heads = 2, 7, 9, 32, 8, 4
    make = lambda *shape, std=1.0, mean=0.0: (torch.randn(shape, generator=gen) * std + mean)
    args = [make(n, h, w, c), make(c, std=0.2, mean=1.0), make(c, std=0.2), make(c, 3 * 64, std=0.2), make(64, c, std=0.2)]
    weight = make(n, h, w, c)
    dev = [a.cuda().requires_grad_() for a in args]
    x, gamma, beta, into, out = dev
    q, k, v = (example.NormAct.apply(x, gamma, beta, ctx, groups).reshape(n, h * w, c) @ into).view(n, h * w, 3, heads, 16).unbind(2)
    y = x + (example.Attend.apply(q, k, v, ctx, False, None, None).reshape(n, h * w, 64) @ out).view(n, h, w, c)
    got = torch.autograd.grad((y * weight.cuda()).sum(), dev)
    ref = [a.double().requires_grad_() for a in args]
    want_y = plain_block(*ref, groups, heads)
    want = torch.autograd.grad((want_y * weight.double()).sum(), ref)
    # sums of up to 64 * 63 products, three one behind the other: 2^12 roundings of the largest numbers that occur
    assert float((y.double().cpu() - want_y).abs().max()) <= 4096 * U * float(want_y.abs().max())
    for g, r in zip(got, want):
        assert float((g.double().cpu() - r).abs().max()) <= 4096 * U * float(r.abs().max())


def test_second_derivatives_are_refused(example, ctx):
    q, k, v = (torch.randn((1, 5, 2, 16), device="cuda").requires_grad_() for _ in range(3))
    first, = torch.autograd.grad(example.Attend.apply(q, k, v, ctx, True, None, None).square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiated again"):
        torch.autograd.grad(first.square().sum(), k)


@pytest.mark.parametrize("clip", [0.0, 0.05])
def test_the_example_with_attention_and_clipping_runs(example, clip):
    history, results = example.main(steps=3, attention=True, clip=clip, report=lambda s: None)
    assert len(history) == 3 and all(x == x for x in history) and results["after"]["images"] == 16


def test_a_recorded_training_step_with_attention_and_clipping(example, ctx):
    """Forward, backward, norm, clipped step in one graph: every replay gives the eager step of the same state."""
    qrm = example.qrm
    gen = torch.Generator("cuda").manual_seed(1)
    make = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    n, l, heads, d = 2, 130, 2, 64
    params = [make(heads * d, heads * d * 3).mul_(0.05), make(heads * d, heads * d).mul_(0.05)]
    x, w = make(n, l, heads * d), make(n, l, heads * d)
    state = [dict(param=p, m=torch.zeros_like(p), v=torch.zeros_like(p)) for p in params]
    opt = qrm.AdamW(ctx, state, torch.float32)
    desc = qrm.attention_desc(n, l, l, heads, heads, d, torch.float32, True, q=(3 * heads * d, d, 0), k=(3 * heads * d, d, 0), v=(3 * heads * d, d, 0))
    qkv, dqkv = torch.empty((n, l, 3, heads, d), device="cuda"), torch.empty((n, l, 3, heads, d), device="cuda")
    o, do, lse = torch.empty((n, l, heads, d), device="cuda"), torch.empty((n, l, heads, d), device="cuda"), torch.empty((n, heads, l), device="cuda")
    grads, norm, scale = [torch.empty_like(p) for p in params], torch.empty(1, device="cuda"), torch.empty(1, device="cuda")

    def step(s):
        torch.mm(x.view(n * l, -1), params[0], out=qkv.view(n * l, -1))
        q, k, v = qkv.unbind(2)
        ctx.qrm_attention(desc, q, k, v, o, lse, None, None, s)
        torch.mm(w.view(n * l, -1), params[1].t(), out=do.view(n * l, -1))          # of the loss sum(w * (o @ params[1]))
        torch.mm(o.view(n * l, -1).t(), w.view(n * l, -1), out=grads[1])
        ctx.qrm_attention_backward(desc, q, k, v, o, do, lse, *dqkv.unbind(2), None, None, s)
        torch.mm(x.view(n * l, -1).t(), dqkv.view(n * l, -1), out=grads[0])
        opt.qrm_adamw_grad_norm(grads, 0.5, norm, scale, None, s)
        opt.qrm_adamw_step(grads, 1, 1e-2, d_grad_scale=scale, stream=s)

    side = torch.cuda.Stream()
    everything = params + [r[k] for r in state for k in ("m", "v")]
    with torch.cuda.stream(side):
        step(side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(side)
    for _ in range(3):
        x.mul_(0.9)
        before = [t.clone() for t in everything]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in everything] + [norm.clone(), scale.clone(), lse.clone()]
        for t, b in zip(everything, before):
            t.copy_(b)
        torch.cuda.synchronize()
        step(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, everything + [norm, scale, lse]))
    opt.close()
