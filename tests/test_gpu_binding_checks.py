"""What the binding of the fine-tuning calls refuses before the library sees it: the C calls get addresses alone."""
import gc
import weakref

import pytest
import torch

pytestmark = pytest.mark.gpu

N, P, C, GROUPS, BITS = 2, 10, 8, 2, 48


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(qrm):
    c = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    yield c
    c.close()


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def test_pitched_maps_beside_dense_descriptors_are_refused(ctx, qrm):
    """A part of the channels of a wider buffer, whose descriptor says that pixels lie side by side: it would be read as if they did."""
    dense, part = zeros(N, P, C), zeros(N, P, C + 4)[:, :, :C]
    stats = zeros(N, GROUPS)
    d = qrm.group_norm_desc(N, P, C, GROUPS, torch.float32)
    for x, y in ((part, dense), (dense, part)):
        with pytest.raises(AssertionError, match="descriptor"):
            ctx.qrm_group_norm(d, x, None, None, y)
    for x, dy, dx in ((part, dense, dense.clone()), (dense, part, dense.clone()), (dense, dense, part)):
        with pytest.raises(AssertionError, match="descriptor"):
            ctx.qrm_group_norm_backward(d, x, dy, None, None, stats, stats, dx)
    torch.cuda.synchronize()


def test_norm_takes_tensors_that_fit_its_descriptor(ctx, qrm):
    x, y, stats, vec = zeros(N, P, C), zeros(N, P, C), zeros(N, GROUPS), zeros(C)
    d = qrm.group_norm_desc(N, P, C, GROUPS, torch.float32)
    ctx.qrm_group_norm(d, x.view(N, 2, 5, C), vec, vec, y.view(N * P, C), stats, stats.clone())
    ctx.qrm_group_norm(d, zeros(N + 1, P, C), zeros(C + 1), None, y.view(-1), zeros(N + 1, GROUPS), stats)
    wide = qrm.group_norm_desc(N, P, C, GROUPS, torch.float32, x_pixel=C + 4)
    ctx.qrm_group_norm(wide, zeros(N, P, C + 4), None, None, y)
    for bad in (dict(x=zeros(N, P, C, dtype=torch.bfloat16)), dict(y=zeros(N, P, C, dtype=torch.float16)), dict(x=zeros(N, P - 1, C)), dict(y=zeros(N - 1, P, C)),
                dict(x=zeros(P, N, C).transpose(0, 1)), dict(gamma=zeros(C - 1)), dict(beta=zeros(C, dtype=torch.float64)), dict(mean=zeros(N, GROUPS - 1)),
                dict(rstd=zeros(N, GROUPS, dtype=torch.bfloat16)), dict(gamma=zeros(2 * C)[::2]), dict(x=torch.zeros(N, P, C))):
        a = dict(dict(x=x, gamma=vec, beta=vec, y=y, mean=stats, rstd=stats), **bad)
        with pytest.raises(AssertionError):
            ctx.qrm_group_norm(d, a["x"], a["gamma"], a["beta"], a["y"], a["mean"], a["rstd"])
    for bad in (dict(dy=zeros(N, P, C, dtype=torch.bfloat16)), dict(dx=zeros(N, P, C - 1)), dict(mean=zeros(GROUPS)), dict(dgamma=zeros(C - 1)),
                dict(dbeta=zeros(C, dtype=torch.bfloat16))):
        a = dict(dict(dy=x, dx=y, mean=stats, dgamma=vec, dbeta=vec), **bad)
        with pytest.raises(AssertionError):
            ctx.qrm_group_norm_backward(d, x, a["dy"], vec, vec, a["mean"], stats, a["dx"], a["dgamma"], a["dbeta"])
    torch.cuda.synchronize()


def test_loss_takes_tensors_that_fit_its_sizes(ctx, qrm):
    good = dict(logits=zeros(N, BITS), target=zeros(BITS, dtype=torch.uint8), rows=1, loss=zeros(1), grad=zeros(N, BITS), bits=zeros(N, dtype=torch.int32),
                symbols=zeros(N, dtype=torch.int32))

    def call(**change):
        a = dict(good, **change)
        ctx.qrm_message_loss(a["logits"], a["target"], a["rows"], N, BITS, 1.0, a["loss"], a["grad"], a["bits"], a["symbols"])

    call()
    call(target=zeros(N, BITS, dtype=torch.bool), rows=N, grad=None, bits=None)
    call(logits=zeros(N + 1, BITS), grad=zeros(N + 1, BITS))
    for bad in (dict(logits=zeros(N, BITS, dtype=torch.float64)), dict(logits=zeros(N - 1, BITS)), dict(target=zeros(BITS)), dict(rows=N), dict(loss=zeros(0)),
                dict(loss=zeros(1, dtype=torch.float64)), dict(grad=zeros(N, BITS - 1)), dict(grad=zeros(N, BITS, dtype=torch.bfloat16)),
                dict(bits=zeros(N, dtype=torch.int64)), dict(symbols=zeros(N - 1, dtype=torch.int32)), dict(logits=zeros(BITS, N).t())):
        with pytest.raises(AssertionError):
            call(**bad)
    torch.cuda.synchronize()


def test_moments_and_scales_have_the_right_types(ctx, qrm):
    codes, scales, out = zeros(300, dtype=torch.int8), zeros(2), zeros(300)
    ctx.qrm_unpack_moment(0, codes, scales, 300, out)
    ctx.qrm_unpack_moment(1, codes.to(torch.uint8), scales, 299, out)
    for a in ((0, codes, scales, 301, out), (0, codes, scales[:1], 300, out), (0, codes, scales, 300, out[:299]), (0, codes.int(), scales, 300, out),
              (0, codes, scales.double(), 300, out)):
        with pytest.raises(AssertionError):
            ctx.qrm_unpack_moment(*a)
    p = zeros(9)
    opt = qrm.AdamW(ctx, [dict(param=p, m=zeros(9), v=zeros(9))], torch.float32)
    opt.qrm_adamw_step([zeros(9)], 1, 0.1, d_grad_scale=torch.ones(1, device="cuda"))
    for scale in (torch.ones(1, dtype=torch.float64, device="cuda"), zeros(0), torch.ones(1)):
        with pytest.raises(AssertionError):
            opt.qrm_adamw_step([zeros(9)], 1, 0.1, d_grad_scale=scale)
    torch.cuda.synchronize()


def test_a_plan_keeps_its_tensors_whatever_becomes_of_the_callers_rows(ctx, qrm):
    """The plan holds addresses: the tensors live as long as it does, also when the caller's dicts are changed or gone."""
    n = 300
    rows = [dict(param=zeros(n), m=zeros(n, dtype=torch.int8), v=zeros(n, dtype=torch.uint8), m_scale=zeros(2), v_scale=zeros(2), copy=zeros(n, dtype=torch.bfloat16)),
            dict(param=zeros(n), m=zeros(n, dtype=torch.int8), v=zeros(n, dtype=torch.uint8), m_scale=zeros(2), v_scale=zeros(2))]
    alive = [weakref.ref(t) for row in rows for t in row.values()]
    opt = qrm.AdamW(ctx, rows, torch.float32)
    rows[0]["m"] = rows[0]["copy"] = None
    rows[0].pop("v_scale")
    rows[1].clear()
    del rows
    gc.collect()
    assert all(r() is not None for r in alive)
    opt.close()
    del opt
    gc.collect()
    assert all(r() is None for r in alive)
