"""What the fine-tuning calls refuse before anything is launched: sizes past a launch, maps written over themselves, moments of other sizes, a first
recorded call.  And sizes at which a launch is cut in another way."""
import ctypes as C

import pytest
import torch

from test_gpu_finetune import check_backward, check_norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as qrm
    return qrm


@pytest.fixture()
def ctx(qrm):
    return qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))


def test_norm_of_more_threads_than_a_launch_has(ctx, qrm):
    x, f = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    p, q = x.data_ptr(), f.data_ptr()
    for N, C_, P in (((1 << 24), 32, 1), ((1 << 31) - 1, 32, 1), (1 << 22, 256, 4)):
        d = qrm.group_norm_desc(N, P, C_, 32, torch.float32)
        assert ctx._lib.qrm_group_norm(ctx._h, C.byref(d), p, None, None, p, None, None, None) == qrm.QRM_E_UNSUPPORTED
        assert ctx._lib.qrm_group_norm_backward(ctx._h, C.byref(d), p, p, None, None, q, q, p, q, None, None) == qrm.QRM_E_UNSUPPORTED


@pytest.mark.parametrize("change,fine", [(dict(y_pixel=9), False), (dict(x_image=40), False), (dict(x_pixel=9, y_pixel=9), True),
                                         (dict(N=1, x_image=40), True), (dict(P=1, x_pixel=9, y_pixel=10, x_image=32, y_image=32), True)])
def test_norm_in_place_needs_equal_strides(ctx, qrm, change, fine):
    buf, f = torch.randn(256, device="cuda"), torch.ones(64, device="cuda")
    other = torch.randn(256, device="cuda")
    d = qrm.group_norm_desc(**dict(dict(N=2, P=4, C=8, groups=2, dtype=torch.float32), **change))
    p, o, q, lib = buf.data_ptr(), other.data_ptr(), f.data_ptr(), ctx._lib
    want = 0 if fine else qrm.QRM_E_INVALID
    assert lib.qrm_group_norm(ctx._h, C.byref(d), p, None, None, p, None, None, None) == want
    assert lib.qrm_group_norm(ctx._h, C.byref(d), p, None, None, o, None, None, None) == 0
    assert lib.qrm_group_norm_backward(ctx._h, C.byref(d), p, o, None, None, q, q, o, None, None, None) == want
    torch.cuda.synchronize()


def test_adamw_limits(ctx, qrm):
    f = torch.zeros(1024, device="cuda")
    q, lib = f.data_ptr(), ctx._lib
    from paper_2509_02447_amd import binding as b
    row = (b._AdamwTensor * 1)()
    for k, v in dict(n=4096 << 24, d_param=q, d_m=q, d_v=q, lr_scale=1.0).items():
        setattr(row[0], k, v)
    out = C.c_void_p()
    assert lib.qrm_adamw_create(ctx._h, C.byref(b._AdamwDesc(1, 0, 0, 1, 32)), row, C.byref(out)) == qrm.QRM_E_UNSUPPORTED and not out.value
    assert lib.qrm_unpack_moment(ctx._h, 0, q, q, 1 << 36, 1, q, None) == qrm.QRM_E_UNSUPPORTED


def test_adamw_takes_moments_of_the_right_sizes_only(ctx, qrm):
    i8, u8 = (torch.zeros(300, dtype=t, device="cuda") for t in (torch.int8, torch.uint8))
    f = torch.zeros(300, device="cuda")
    s = torch.zeros(2, device="cuda")
    good8, good32 = dict(param=f, m=i8, v=u8, m_scale=s, v_scale=s.clone()), dict(param=f, m=f.clone(), v=f.clone())
    for good in (good8, good32):
        qrm.AdamW(ctx, [good], torch.float32).close()
    for good, change in ((good8, dict(v=i8)), (good8, dict(m=i8[:299])), (good8, dict(m_scale=s[:1])), (good8, dict(v_scale=s.half())),
                         (good32, dict(v=u8)), (good32, dict(v=f[:299])), (good32, dict(copy=f[:299].bfloat16()))):
        with pytest.raises(AssertionError):
            qrm.AdamW(ctx, [dict(good, **change)], torch.float32)


def test_first_recorded_loss_is_refused(ctx, qrm):
    """A loss of several workgroups counts them in memory that its stream's first call clears: that call is not recorded, the next may be."""
    N = 4096
    g = torch.Generator().manual_seed(3)
    logits = torch.randn((N, 48), generator=g).cuda()
    target = (torch.rand((N, 48), generator=g) < 0.5).to(torch.uint8).cuda()
    eager, loss = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ctx.qrm_message_loss(logits, target, N, N, 48, 1.0, eager)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        ctx.qrm_group_norm(qrm.group_norm_desc(4, 4096, 64, 8, torch.float32), torch.zeros(4, 4096, 64, device="cuda"), None, None,
                           torch.zeros(4, 4096, 64, device="cuda"), stream=stream)  # (the stream's workspace is there, its counters are not)
        torch.cuda.synchronize()
        graph.capture_begin(capture_error_mode="relaxed")
        with pytest.raises(RuntimeError, match="recorded"):
            ctx.qrm_message_loss(logits, target, N, N, 48, 1.0, loss, stream=stream)
        loss.zero_()
        graph.capture_end()
        ctx.qrm_message_loss(logits, target, N, N, 48, 1.0, loss, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(loss, eager)
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin(capture_error_mode="relaxed")
        ctx.qrm_message_loss(logits, target, N, N, 48, 1.0, loss, stream=stream)
        graph.capture_end()
        for _ in range(3):
            loss.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(loss, eager)


@pytest.mark.parametrize("workgroups", [5, 15, 16, 17, 31, 33, 100, 255, 256, 300])
def test_loss_counts_every_workgroup(ctx, workgroups):
    """64 images of 12 symbols to a workgroup, the last one not full.  All terms are positive: a relative bound of the 48 additions of an image,
    a logit's functions (four roundings, a unit of each of three) and two roundings of the mean: under 80 half units of 32 bits."""
    N = 64 * workgroups - 7
    g = torch.Generator().manual_seed(workgroups)
    logits = 3 * torch.randn((N, 48), generator=g)
    target = (torch.rand((N, 48), generator=g) < 0.5).to(torch.uint8)
    want = torch.nn.functional.binary_cross_entropy_with_logits(logits.double(), target.double()).item()
    dev, dev_target, loss = logits.cuda(), target.cuda(), torch.zeros(3, device="cuda")
    for i in range(3):  # (the counts are left as they were found)
        ctx.qrm_message_loss(dev, dev_target, N, N, 48, 0.0, loss[i:i + 1])
    got = loss.cpu()
    assert torch.equal(got[1:], got[:2])
    assert abs(got[0].item() - want) <= 80 * 2.0 ** -24 * want


# images, pixels, channels, groups: tiles of a part of a line, in numbers that eight dies divide or not; a few more tiles than compute units; one round of
# workgroups, one and a bit, one and a half
CUTS = [(1, 100, 488, 61), (3, 100, 512, 32), (5, 33, 520, 65), (13, 70, 72, 9), (16, 200, 512, 32), (17, 300, 512, 32), (20, 1030, 256, 16), (33, 40, 512, 32),
        (48, 1025, 256, 8), (270, 9, 32, 4), (600, 17, 40, 5)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,p,c,groups", CUTS)
def test_norm_however_it_is_cut(ctx, qrm, n, p, c, groups, dtype):
    check_norm(ctx, qrm, n, p, c, groups, dtype, "silu", seed=n + p)
    check_backward(ctx, qrm, n, p, c, groups, dtype, "silu", seed=n + p)


def test_norm_past_the_caches_in_one_launch(ctx, qrm):
    check_norm(ctx, qrm, 64, 601, 512, 32, torch.bfloat16, "silu", seed=5)
