"""The norm of all gradients with the factor that clips it, and gradients times a factor, on the GPU against 64 bits (oracle/attention.py).

Squares and sums are taken in 64 bits, so the norm and the factor are off by the rounding to 32 bits they are returned in: u = 2^-24 of their value, and
2^-40 for sums of up to 2^13 numbers one after the other; a scaled gradient by the factor's rounding, the product's and the type's.
"""
import numpy as np
import pytest
import torch

from oracle import attention as at

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(qrm):
    c = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def plan(qrm, ctx, sizes, dtype):
    rows = [dict(param=torch.zeros(n, device="cuda"), m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda")) for n in sizes]
    return qrm.AdamW(ctx, rows, dtype)


def gradients(sizes, dtype, seed=0, level=1.0, shift=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.cat([torch.zeros(shift), torch.randn(n, generator=g) * level]).to(dtype).cuda()[shift:] for n in sizes]


def check(qrm, ctx, sizes, dtype, max_norm=1.0, unscale=None, missing=(), **kw):
    opt, grads = plan(qrm, ctx, sizes, dtype), gradients(sizes, dtype, **kw)
    grads = [None if i in missing else g for i, g in enumerate(grads)]
    norm, scale = torch.full((1,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    by = None if unscale is None else torch.full((1,), unscale, device="cuda")
    opt.qrm_adamw_grad_norm(grads, max_norm, norm, scale, by)
    outs = [None if g is None else torch.full_like(g, 7.0) for g in grads]
    opt.qrm_adamw_scale_grads(grads, scale, outs)
    torch.cuda.synchronize()
    want, part = at.grad_norm([None if g is None else f64(g) for g in grads], max_norm, 1.0 if by is None else float(by))
    assert abs(float(norm) - want) <= (U + 2.0 ** -40) * want
    assert abs(float(scale) - part) <= (U + 2.0 ** -40) * part
    for g, o in zip(grads, outs):
        if g is not None:
            w = f64(g) * part
            assert (np.abs(f64(o) - w) <= (HALF[dtype] + 2.01 * U) * np.abs(w) + TINY[dtype]).all()
    before = [None if o is None else o.clone() for o in outs]
    opt.qrm_adamw_scale_grads(grads, scale)                           # in place
    torch.cuda.synchronize()
    assert all(g is None or torch.equal(g, b) for g, b in zip(grads, before))
    opt.close()


# no elements, one, pieces of 4096 less and more one, one workgroup's pieces and one more, all workgroups', more tensors than one launch names (448; 224 with outputs)
SIZES = [[0], [1], [4095, 4096, 4097], [1, 0, 3, 5, 7, 0], [4096 * 64], [4096 * 64 + 1], [4096 * 70 + 33] * 3, [100003, 5, 40000, 262144], [3_000_001], [17] * 500, [1000 + i for i in range(900)],
         [33] * 224, [33] * 225, [33] * 448, [33] * 449]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_sizes(qrm, ctx, which, dtype):
    check(qrm, ctx, SIZES[which], dtype, seed=which)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_factors(qrm, ctx, dtype):
    for max_norm, unscale, level in ((1.0, None, 1e-3), (0.25, 0.125, 1.0), (1e6, 2.0, 1.0), (np.inf, 0.5, 3.0), (1e-3, 1.0, 1.0), (2.0, 1e-4, 100.0)):
        check(qrm, ctx, [5000, 333, 12288], dtype, max_norm, unscale, level=level)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("shift", [1, 2, 4, 8])
def test_alignment(qrm, ctx, shift, dtype):
    check(qrm, ctx, [9001, 4096, 31], dtype, shift=shift)


def test_tensors_without_a_gradient(qrm, ctx):
    check(qrm, ctx, [100, 5000, 1, 9000], torch.bfloat16, missing=(1, 2))
    check(qrm, ctx, [100, 5000], torch.float32, missing=(0, 1))
    check(qrm, ctx, [50] * 460, torch.float32, missing=range(440, 460))
    check(qrm, ctx, [], torch.float32)


def test_squares_outside_32_bits(qrm, ctx):
    check(qrm, ctx, [100, 100000], torch.float32, level=1e30)
    check(qrm, ctx, [100, 100000], torch.float32, level=1e-30)


def test_one_large_among_many_small(qrm, ctx):
    opt = plan(qrm, ctx, [1_000_000, 1], torch.float32)
    grads = [torch.full((1_000_000,), 1e-4, device="cuda"), torch.full((1,), 1000.0, device="cuda")]
    norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    opt.qrm_adamw_grad_norm(grads, 10.0, norm, scale)
    torch.cuda.synchronize()
    want, part = at.grad_norm([f64(g) for g in grads], 10.0)
    assert abs(float(norm) - want) <= (U + 2.0 ** -40) * want and abs(float(scale) - part) <= (U + 2.0 ** -40) * part
    opt.close()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_gradients_that_are_not_finite(qrm, ctx, bad):
    sizes = [5000, 70000]
    opt, grads = plan(qrm, ctx, sizes, torch.float32), gradients(sizes, torch.float32)
    grads[1][69999] = bad
    norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    opt.qrm_adamw_grad_norm(grads, 1.0, norm, scale)
    torch.cuda.synchronize()
    if np.isnan(bad):
        assert bool(torch.isnan(norm)) and bool(torch.isnan(scale))
    else:
        assert float(norm) == np.inf and float(scale) == 0.0
    opt.close()


def test_a_clipped_step(qrm, ctx):
    """What the norm leaves is what a step takes: a clipped step is the step of the scaled gradients."""
    sizes = [5000, 333, 20000]
    state = [[torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)) for n in sizes] for _ in range(2)]
    results = []
    for fused, params in zip((True, False), state):
        rows = [dict(param=p, m=torch.zeros_like(p), v=torch.zeros_like(p)) for p in params]
        opt, grads = qrm.AdamW(ctx, rows, torch.float32), gradients(sizes, torch.float32, seed=1)
        norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
        opt.qrm_adamw_grad_norm(grads, 0.5, norm, scale)
        if not fused:
            opt.qrm_adamw_scale_grads(grads, scale)
        opt.qrm_adamw_step(grads, 1, 1e-2, d_grad_scale=scale if fused else None)
        torch.cuda.synchronize()
        results.append([p.clone() for p in params] + [r["m"] for r in rows] + [r["v"] for r in rows])
        opt.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_the_same_bits_on_other_streams_and_in_graphs(qrm, ctx):
    sizes = [4096 * 300 + 5, 77, 1_000_000]
    opt, grads = plan(qrm, ctx, sizes, torch.bfloat16), gradients(sizes, torch.bfloat16)
    outs = [torch.empty_like(g) for g in grads]
    def call(norm, scale, s):
        opt.qrm_adamw_grad_norm(grads, 1.0, norm, scale, None, s)
        opt.qrm_adamw_scale_grads(grads, scale, outs, s)
    new = lambda: (torch.empty(1, device="cuda"), torch.empty(1, device="cuda"))
    first = new()
    call(*first, None)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), new()
    call(*other, side)
    side.synchronize()
    assert torch.equal(first[0], other[0]) and torch.equal(first[1], other[1])
    graph, held = torch.cuda.CUDAGraph(), new()
    with torch.cuda.graph(graph, stream=side):
        call(*held, side)
    for k in range(3):
        for g in grads:
            g.mul_(0.5 if k else 1.0)
        eager = new()
        call(*eager, None)
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for t in held + tuple(outs):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], eager[0]) and torch.equal(held[1], eager[1]) and all(torch.equal(a, b) for a, b in zip(outs, want))
    opt.close()


def test_refusals(qrm, ctx):
    opt, grads = plan(qrm, ctx, [10, 20], torch.float32), gradients([10, 20], torch.float32)
    norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    outs = [torch.empty_like(g) for g in grads]

    def refused(call, status=qrm.QRM_E_INVALID):
        with pytest.raises(qrm.QrmError) as e:
            call()
        assert e.value.status == status and e.value.message

    for bad in (0.0, -1.0, np.nan):
        refused(lambda: opt.qrm_adamw_grad_norm(grads, bad, norm, scale))
    refused(lambda: opt.qrm_adamw_grad_norm(grads, 1.0, None, None))
    refused(lambda: opt.qrm_adamw_grad_norm(grads, 1.0, norm, norm))
    refused(lambda: opt.qrm_adamw_grad_norm(grads, 1.0, norm, scale, scale))
    refused(lambda: opt.qrm_adamw_scale_grads(grads, None, outs))
    refused(lambda: opt.qrm_adamw_scale_grads(grads, scale, [outs[0], None]))
    refused(lambda: opt.qrm_adamw_scale_grads([grads[0], None], scale, outs))
    for wrong in ([grads[0]], [grads[0], grads[1][:5]], [grads[0].bfloat16(), grads[1]], [grads[0], grads[1].cpu()]):
        with pytest.raises(AssertionError):
            opt.qrm_adamw_grad_norm(wrong, 1.0, norm, scale)
        with pytest.raises(AssertionError):
            opt.qrm_adamw_scale_grads(grads, scale, wrong)
    lib = ctx._lib
    assert lib.qrm_adamw_grad_norm(ctx._h, None, None, 1.0, None, norm.data_ptr(), None, None) == qrm.QRM_E_INVALID
    assert lib.qrm_adamw_grad_norm(ctx._h, opt._h, None, 1.0, None, norm.data_ptr(), None, None) == qrm.QRM_E_INVALID
    assert lib.qrm_adamw_grad_norm(ctx._h, opt._h, opt._pointers(grads), 1.0, None, norm.data_ptr() + 2, None, None) == qrm.QRM_E_INVALID
    assert lib.qrm_adamw_scale_grads(ctx._h, opt._h, opt._pointers(grads), scale.data_ptr(), None, None) == qrm.QRM_E_INVALID
    opt.close()
