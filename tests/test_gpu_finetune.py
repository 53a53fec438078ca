"""The fine-tuning operators on the GPU, through the C ABI, against the 64-bit oracle (oracle/finetune.py).

Tolerances come from the number formats: u = 2^-24 is half a unit in the last place of 32 bits, `half` that of the output's type.  Sums run
over at most 128 numbers one after the other and in trees beyond, so a mean is within 128 u of the largest value; the rest are a handful
of roundings.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import finetune as ft

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
EPS = 1e-6
CODE = dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1)


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(qrm):
    c = qrm.Context(rs=CODE)
    yield c
    c.close()


def f64(t):
    return t.detach().double().cpu().numpy()


def padded(shape, dtype, gap_pixel=0, gap_image=0, shift=0, fill=7.0):
    """A map [N,P,C] inside a larger buffer: `shift` elements in, `gap`s behind pixels and images."""
    n, p, c = shape
    xp, xn = c + gap_pixel, p * (c + gap_pixel) + gap_image
    buf = torch.full((shift + n * xn + 64,), fill, dtype=dtype, device="cuda")
    return buf, buf.as_strided(shape, (xn, xp, 1), shift)


def desc_of(qrm, x, y, groups, act, eps=EPS):
    n, p, c = x.shape
    return qrm.group_norm_desc(n, p, c, groups, x.dtype, act, eps, x.stride(1), x.stride(0), y.stride(1), y.stride(0))


# ---------------------------------------------------------------- group norm

# pixels, channels, groups: single pixels, odd ones, one more and less than what a workgroup's rows hold, channels that no piece of 16, 8 or
# 4 bytes divides, groups of one channel, one group, groups that straddle pieces, groups wider than a workgroup of 256 pieces
SHAPES = [(1, 4, 4), (1, 8, 2), (1, 64, 32), (2, 6, 2), (3, 5, 1), (17, 1, 1), (63, 64, 32), (64, 96, 8), (65, 60, 12), (257, 12, 12),
          (1000, 32, 4), (333, 512, 32), (5, 1020, 12), (7, 1001, 7), (9, 2048, 1), (4, 4096, 2), (130, 130, 13), (4099, 24, 3)]


def check_norm(ctx, qrm, n, p, c, groups, dtype, act, seed, gaps=(0, 0, 0), affine=True, level=1.0, spread=2.0, in_place=False, stats=True):
    g = torch.Generator().manual_seed(seed)
    src, x = padded((n, p, c), dtype, *gaps)
    x.copy_((torch.randn((n, p, c), generator=g) * spread + level).to(dtype))
    gamma = (torch.randn(c, generator=g) * 0.3 + 1.0).cuda() if affine else None
    beta = (torch.randn(c, generator=g) * 0.3).cuda() if affine else None
    given = f64(x)
    dst, y = (src, x) if in_place else padded((n, p, c), dtype, gaps[0] // 2, gaps[1], gaps[2])
    mean = torch.full((n, groups), np.nan, device="cuda") if stats else None
    rstd = torch.full((n, groups), np.nan, device="cuda") if stats else None
    ctx.qrm_group_norm(desc_of(qrm, x, y, groups, act), x, gamma, beta, y, mean, rstd)
    torch.cuda.synchronize()
    ry, rm, rr = ft.group_norm(given, None if gamma is None else f64(gamma), None if beta is None else f64(beta), groups, act, EPS)
    big = np.abs(given.reshape(n, p, groups, -1)).max(axis=(1, 3))
    if stats:
        assert (np.abs(f64(mean) - rm) <= 128 * U * big).all()
        # the mean's error and each value's rounding against the spread, squared sums' errors of their own
        assert (np.abs(f64(rstd) / rr - 1) <= 128 * U * (1 + big * rr)).all()
    h = np.abs((given - np.repeat(rm, c // groups, 1)[:, None]) * np.repeat(rr, c // groups, 1)[:, None])
    off = 128 * U * (h + np.repeat(big * rr, c // groups, 1)[:, None]) * (1 if gamma is None else np.abs(f64(gamma))) + 8 * U * (0 if beta is None else np.abs(f64(beta)))
    z = np.abs(ry) + off
    tol = (1.2 + z) * off + (8 + z) * U * np.abs(ry) + HALF[dtype] * (np.abs(ry) + off) + TINY[dtype]  # (the steepest slope of z sigmoid(z) is 1.1)
    err = np.abs(f64(y) - ry)
    assert (err <= tol).all(), f"off by {(err / tol).max()} of what is allowed"
    if not in_place:  # nothing else of the buffer was written
        y.fill_(7.0)
        assert bool((dst == 7.0).all())
    return x, gamma, beta, rm, rr


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("p,c,groups", SHAPES)
def test_group_norm_shapes(ctx, qrm, p, c, groups, dtype):
    for k, act in enumerate(("silu", "relu", "none")):
        check_norm(ctx, qrm, 1 + k, p, c, groups, dtype, act, seed=p * 7 + c + k, affine=k != 1 or p % 2 == 0, stats=k != 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gaps", [(8, 0, 0), (1, 0, 0), (0, 3, 0), (0, 0, 1), (2, 6, 2), (4, 8, 4), (300, 17, 3)])
def test_group_norm_strides_and_alignment(ctx, qrm, gaps, dtype):
    check_norm(ctx, qrm, 3, 100, 64, 16, dtype, "silu", seed=sum(gaps), gaps=gaps)
    check_norm(ctx, qrm, 2, 37, 300, 1, dtype, "none", seed=sum(gaps), gaps=gaps)


@pytest.mark.parametrize("n,p,c,groups", [(1, 65536, 32, 8), (2, 40000, 128, 32), (70, 64, 32, 4), (1, 200000, 3, 1), (1, 16384, 512, 32)])
def test_group_norm_large_maps(ctx, qrm, n, p, c, groups):
    check_norm(ctx, qrm, n, p, c, groups, torch.bfloat16, "silu", seed=n + p)


@pytest.mark.parametrize("level,spread", [(1000.0, 1.0), (1e-6, 1e-8), (1e12, 1e10), (-300.0, 0.01), (5.0, 0.0)])
def test_group_norm_levels_far_from_zero(ctx, qrm, level, spread):
    check_norm(ctx, qrm, 2, 777, 40, 5, torch.float32, "none", seed=11, level=level, spread=spread)


def test_group_norm_one_pixel_far_from_all_others(ctx, qrm):
    x = torch.randn((1, 4000, 16), generator=torch.Generator().manual_seed(1)).add_(500.0)
    x[0, 0] = 0.0                                            # (sums taken about the first pixel would cancel)
    y = torch.empty_like(x, device="cuda")
    mean, rstd = torch.empty((1, 4), device="cuda"), torch.empty((1, 4), device="cuda")
    ctx.qrm_group_norm(qrm.group_norm_desc(1, 4000, 16, 4, x.dtype), x.cuda(), None, None, y, mean, rstd)
    ry, rm, rr = ft.group_norm(f64(x), None, None, 4, "none", EPS)
    assert (np.abs(f64(mean) - rm) <= 128 * U * 505).all() and (np.abs(f64(rstd) / rr - 1) <= 128 * U * (1 + 505 * rr)).all()


@pytest.mark.parametrize("in_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,p,c,groups", [(2, 50, 64, 8), (1, 30000, 96, 8)])
def test_group_norm_in_place(ctx, qrm, n, p, c, groups, in_dtype):
    check_norm(ctx, qrm, n, p, c, groups, in_dtype, "silu", seed=5, in_place=True, gaps=(8, 0, 0))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("p", [40, 20000])
def test_group_norm_values_that_are_not_finite_stay_in_their_group(ctx, qrm, bad, p):
    n, c, groups = 2, 32, 4
    g = torch.Generator().manual_seed(3)
    clean = torch.randn((n, p, c), generator=g)
    dirty = clean.clone()
    dirty[1, p - 3, 17] = bad                                # group 2 of image 1
    gamma, beta = torch.rand(c, generator=g).cuda(), torch.rand(c, generator=g).cuda()
    dy = torch.randn((n, p, c), generator=g).cuda()
    for act in ("silu", "relu", "none"):
        out = []
        for x in (clean.cuda(), dirty.cuda()):
            y, dx = torch.empty_like(x), torch.empty_like(x)
            mean, rstd = torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
            dgamma, dbeta = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
            d = qrm.group_norm_desc(n, p, c, groups, x.dtype, act)
            ctx.qrm_group_norm(d, x, gamma, beta, y, mean, rstd)
            ctx.qrm_group_norm_backward(d, x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta)
            out.append([t.cpu() for t in (y, dx, mean, rstd, dgamma, dbeta)])
        (y0, dx0, m0, r0, dg0, db0), (y1, dx1, m1, r1, dg1, db1) = out
        hit = torch.zeros((n, p, c), dtype=torch.bool)
        hit[1, :, 16:24] = True
        for a, b in ((y0, y1), (dx0, dx1)):
            assert torch.equal(a[~hit], b[~hit]) and bool(torch.isnan(b[hit]).all())
        assert bool(torch.isnan(dg1[16:24]).all())
        rest = torch.arange(c)[(torch.arange(c) < 16) | (torch.arange(c) >= 24)]
        assert torch.equal(dg0[rest], dg1[rest]) and torch.equal(db0[rest], db1[rest])


def test_group_norm_images_more_than_2_31_elements_apart(ctx, qrm):
    far = (1 << 31) + 64
    buf = torch.empty(2 * far, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, 30, 64), (far, 64, 1))
    x.copy_(torch.randn((2, 30, 64), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16))
    dy = torch.randn((2, 30, 64), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    near = x.contiguous()
    got = []
    for t in (x, near):
        y, dx = t.as_strided(t.shape, t.stride(), 64 * 40) if t is x else torch.empty_like(t), torch.empty_like(near)
        y = buf.as_strided((2, 30, 64), (far, 64, 1), 64 * 40) if t is x else torch.empty_like(near)
        mean, rstd = torch.empty((2, 8), device="cuda"), torch.empty((2, 8), device="cuda")
        ctx.qrm_group_norm(desc_of(qrm, t, y, 8, "silu"), t, None, None, y, mean, rstd)
        d = qrm.group_norm_desc(2, 30, 64, 8, t.dtype, "silu", EPS, t.stride(1), t.stride(0))
        dxs = buf.as_strided((2, 30, 64), (far, 64, 1), 64 * 80) if t is x else dx
        dgamma, dbeta = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
        ctx.qrm_group_norm_backward(d, t, dy, None, None, mean, rstd, dxs, dgamma, dbeta)
        got.append([v.contiguous().cpu() for v in (y, mean, rstd, dxs, dgamma, dbeta)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


# ---------------------------------------------------------------- group norm, backward

def check_backward(ctx, qrm, n, p, c, groups, dtype, act, seed, gaps=(0, 0, 0), affine=True, wanted=("dx", "dgamma", "dbeta"), in_place=False, repeat=False):
    x, gamma, beta, rm, rr = check_norm(ctx, qrm, n, p, c, groups, dtype, act, seed, gaps, affine)
    mean, rstd = torch.from_numpy(rm).float().cuda(), torch.from_numpy(rr).float().cuda()
    g = torch.Generator().manual_seed(seed + 1)
    _, dy = padded((n, p, c), dtype, gaps[0] if in_place else gaps[0] // 2, gaps[1], gaps[2])
    dy.copy_(torch.randn((n, p, c), generator=g).to(dtype))
    given = f64(dy)
    buf, dx = (None, dy) if in_place else padded((n, p, c), dtype, *gaps)
    out = dict(dx=dx if "dx" in wanted else None, dgamma=torch.full((c,), np.nan, device="cuda") if "dgamma" in wanted else None,
               dbeta=torch.full((c,), np.nan, device="cuda") if "dbeta" in wanted else None)
    d = desc_of(qrm, x, dy, groups, act)
    ctx.qrm_group_norm_backward(d, x, dy, gamma, beta, mean, rstd, out["dx"], out["dgamma"], out["dbeta"])
    torch.cuda.synchronize()
    xs = f64(x)
    gm, bt = np.ones(c) if gamma is None else f64(gamma), np.zeros(c) if beta is None else f64(beta)
    rdx, rdg, rdb = ft.group_norm_backward(xs, given, gm, bt, f64(mean), f64(rstd), groups, act)
    wide = lambda v: np.repeat(v, c // groups, 1)[:, None, :]
    h = (xs - wide(f64(mean))) * wide(f64(rstd))
    z = np.abs(gm * h) + np.abs(bt)
    dz = np.abs(given) * (1.2 if act == "silu" else 1.0)
    slip = dz * (16 + 4 * z) * U                              # of dz: the activation's slope and its argument
    if act == "relu":                                         # z within rounding of zero: either slope
        slip = slip + np.where(np.abs(gm * h + bt) <= 4 * U * z, np.abs(given), 0.0)
    size_b, size_g = dz.sum(axis=(0, 1)), (dz * np.abs(h)).sum(axis=(0, 1))
    if "dbeta" in wanted:
        assert (np.abs(f64(out["dbeta"]) - rdb) <= slip.sum(axis=(0, 1)) + 128 * U * size_b + 1e-30).all()
    if "dgamma" in wanted:
        assert (np.abs(f64(out["dgamma"]) - rdg) <= (slip * np.abs(h)).sum(axis=(0, 1)) + 132 * U * size_g + 1e-30).all()
    if "dx" in wanted:
        over = lambda v: wide(v.reshape(n, p, groups, -1).mean(axis=(1, 3)))
        a, b = np.abs(gm) * dz, np.abs(gm) * dz * np.abs(h)
        tol = wide(f64(rstd)) * (np.abs(gm) * slip + over(np.abs(gm) * slip) + np.abs(h) * over(np.abs(gm) * slip * np.abs(h)) +
                                 140 * U * (a + over(a) + np.abs(h) * over(b)))
        err = np.abs(f64(dx) - rdx)
        tol = tol + HALF[dtype] * (np.abs(rdx) + tol) + TINY[dtype]
        assert (err <= tol).all(), f"off by {(err / tol).max()} of what is allowed"
        if not in_place:
            dx.fill_(7.0)
            assert bool((buf == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("p,c,groups", SHAPES)
def test_group_norm_backward_shapes(ctx, qrm, p, c, groups, dtype):
    for k, act in enumerate(("silu", "relu", "none")):
        check_backward(ctx, qrm, 1 + k, p, c, groups, dtype, act, seed=p * 3 + c + k, affine=k != 1 or p % 2 == 0)


@pytest.mark.parametrize("gaps", [(8, 0, 0), (2, 6, 2), (0, 0, 1), (300, 17, 3)])
def test_group_norm_backward_strides_and_alignment(ctx, qrm, gaps):
    check_backward(ctx, qrm, 3, 100, 64, 16, torch.bfloat16, "silu", seed=sum(gaps), gaps=gaps)
    check_backward(ctx, qrm, 2, 37, 300, 1, torch.float32, "relu", seed=sum(gaps), gaps=gaps)


@pytest.mark.parametrize("n,p,c,groups", [(1, 65536, 32, 8), (2, 40000, 128, 32), (70, 64, 32, 4), (1, 200000, 3, 1), (1, 16384, 512, 32)])
def test_group_norm_backward_large_maps(ctx, qrm, n, p, c, groups):
    check_backward(ctx, qrm, n, p, c, groups, torch.bfloat16, "silu", seed=n + p)


@pytest.mark.parametrize("n,p", [(3, 40), (2, 9000)])
@pytest.mark.parametrize("wanted", [("dx",), ("dgamma",), ("dbeta", "dgamma"), ("dx", "dbeta")])
def test_group_norm_backward_outputs_that_are_not_wanted(ctx, qrm, wanted, n, p):
    check_backward(ctx, qrm, n, p, 48, 6, torch.float32, "silu", seed=9, wanted=wanted)


@pytest.mark.parametrize("n,p", [(3, 40), (2, 30000)])
def test_group_norm_backward_in_place_of_dy(ctx, qrm, n, p):
    check_backward(ctx, qrm, n, p, 64, 8, torch.bfloat16, "silu", seed=4, in_place=True, gaps=(8, 0, 0))


def test_group_norm_backward_of_groups_of_one_value_is_zero(ctx, qrm):
    c = 40
    x, dy = torch.randn((3, 1, c)).cuda(), torch.randn((3, 1, c)).cuda()
    mean, rstd, y, dx = torch.empty((3, c), device="cuda"), torch.empty((3, c), device="cuda"), torch.empty_like(x), torch.full_like(x, 9.0)
    gamma, beta = torch.randn(c).cuda(), torch.randn(c).cuda()
    d = qrm.group_norm_desc(3, 1, c, c, x.dtype, "silu")
    ctx.qrm_group_norm(d, x, gamma, beta, y, mean, rstd)
    ctx.qrm_group_norm_backward(d, x, dy, gamma, beta, mean, rstd, dx, torch.empty(c, device="cuda"), None)
    assert torch.equal(mean, x[:, 0]) and not bool(dx.any())
    assert torch.allclose(y, (beta * torch.sigmoid(beta)).expand(3, 1, c), rtol=1e-6, atol=0)


@pytest.mark.parametrize("p", [30, 9000])
def test_group_norm_same_bits_again_on_other_streams_and_beside_other_work(ctx, qrm, p):
    n, c, groups = 3, 96, 8
    g = torch.Generator().manual_seed(8)
    x, dy = (torch.randn((n, p, c), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    gamma, beta = torch.rand(c, generator=g).cuda(), torch.rand(c, generator=g).cuda()
    d = qrm.group_norm_desc(n, p, c, groups, x.dtype, "silu")

    def once():
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd, dgamma, dbeta = (torch.empty(s, device="cuda") for s in ((n, groups), (n, groups), (c,), (c,)))
        ctx.qrm_group_norm(d, x, gamma, beta, y, mean, rstd)
        ctx.qrm_group_norm_backward(d, x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta)
        return y, mean, rstd, dx, dgamma, dbeta

    first = once()
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(once())
    torch.cuda.synchronize()
    for s in streams:
        ctx.qrm_release_stream(s)
    assert all(torch.equal(a, b) for out in got for a, b in zip(first, out))


@pytest.mark.parametrize("c,groups,dtype", [(8192, 1, torch.bfloat16), (8192, 2, torch.float32), (1024, 1, torch.float32), (6144, 1, torch.float16), (513, 1, torch.float32)])
def test_group_norm_wide_groups(ctx, qrm, c, groups, dtype):
    for p in (5, 64, 700):
        check_backward(ctx, qrm, 2, p, c, groups, dtype, "silu", seed=c + p)


@pytest.mark.parametrize("n,p,c,groups", [(300, 40, 64, 8), (64, 512, 256, 32), (33, 2048, 512, 32), (2000, 1, 32, 32), (1, 65, 512, 32), (7, 1025, 128, 32)])
def test_group_norm_between_one_launch_and_two(ctx, qrm, n, p, c, groups):
    """Sizes on both sides of the rules that give a tile to one workgroup, and tiles of half a line to few images."""
    if n * p * c < 5_000_000:
        check_backward(ctx, qrm, n, p, c, groups, torch.bfloat16, "silu", seed=n + p)
    else:                                                    # too large for the 64-bit oracle in a test: image by image the same bits
        g = torch.Generator().manual_seed(n)
        x, dy = (torch.randn((n, p, c), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
        d = qrm.group_norm_desc(n, p, c, groups, x.dtype, "silu")
        ctx.qrm_group_norm(d, x, None, None, y, mean, rstd)
        ctx.qrm_group_norm_backward(d, x, dy, None, None, mean, rstd, dx)
        torch.cuda.synchronize()
        for i in (0, n // 2, n - 1):
            ry, rm, rr = ft.group_norm(f64(x[i:i + 1]), None, None, groups, "silu", EPS)
            rdx = ft.group_norm_backward(f64(x[i:i + 1]), f64(dy[i:i + 1]), None, None, rm, rr, groups, "silu")[0]
            # a group's mean and spread are near 0 and 1 here: the errors of check_norm and check_backward, at their largest
            assert (np.abs(f64(y[i]) - ry[0]) <= HALF[x.dtype] * np.abs(ry[0]) + 1000 * U).all()
            assert (np.abs(f64(dx[i]) - rdx[0]) <= HALF[x.dtype] * np.abs(rdx[0]) + 4000 * U).all()


def test_more_streams_than_workspaces(ctx, qrm):
    """A stream not seen before takes over a workspace that a call has just used on another one."""
    n, p, c, groups = 2, 9000, 64, 8
    g = torch.Generator().manual_seed(12)
    maps = [torch.randn((n, p, c), generator=g).to(torch.bfloat16).cuda() for _ in range(4)]
    d = qrm.group_norm_desc(n, p, c, groups, torch.bfloat16, "silu")

    def once(x):
        y, mean, rstd = torch.empty_like(x), torch.empty((n, groups), device="cuda"), torch.empty((n, groups), device="cuda")
        dx, dgamma = torch.empty_like(x), torch.empty(c, device="cuda")
        ctx.qrm_group_norm(d, x, None, None, y, mean, rstd)
        ctx.qrm_group_norm_backward(d, x, y, None, None, mean, rstd, dx, dgamma)
        return y, mean, rstd, dx, dgamma

    expected = [once(x) for x in maps]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2 * qrm.QRM_MAX_STREAMS + 3)], []
    for i in range(3 * len(streams)):
        with torch.cuda.stream(streams[i % len(streams)]):
            got.append(once(maps[i % 4]))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(expected[i % 4], out)), i
    for s in streams:
        ctx.qrm_release_stream(s)


def test_group_norm_no_images(ctx, qrm):
    x = torch.empty((0, 10, 8), device="cuda")
    d = qrm.group_norm_desc(0, 10, 8, 2, x.dtype)
    dgamma, dbeta = torch.full((8,), 3.0, device="cuda"), torch.full((8,), 3.0, device="cuda")
    empty = torch.empty((0, 2), device="cuda")
    ctx.qrm_group_norm(d, x, None, None, x, empty, empty)
    ctx.qrm_group_norm_backward(d, x, x, None, None, empty, empty, x, dgamma, dbeta)
    assert not bool(dgamma.any()) and not bool(dbeta.any())


def test_group_norm_refusals(ctx, qrm):
    lib, h = ctx._lib, ctx._h
    x, f = torch.zeros((2, 4, 8), device="cuda"), torch.zeros(64, device="cuda")
    good = dict(N=2, P=4, C=8, groups=2, dtype=torch.float32, act="none", eps=1e-6)

    def call(change=None, field=None, value=None, x_=None, y=None, mean=None, rstd=None):
        d = qrm.group_norm_desc(**dict(good, **(change or {})))
        if field:
            setattr(d, field, value)
        p = x.data_ptr()
        return lib.qrm_group_norm(h, C.byref(d), p if x_ is None else x_, None, None, p if y is None else y, mean, rstd, None)

    assert call() == 0
    for kw in (dict(change=dict(N=-1)), dict(change=dict(P=0)), dict(change=dict(groups=3)), dict(change=dict(groups=0)), dict(change=dict(C=0)),
               dict(field="type", value=3), dict(field="act", value=-1), dict(change=dict(eps=0.0)), dict(change=dict(eps=float("nan"))),
               dict(change=dict(x_pixel=7)), dict(change=dict(y_pixel=-8)), dict(change=dict(x_image=31)), dict(change=dict(y_image=-1)),
               dict(change=dict(x_image=1 << 62)), dict(change=dict(x_pixel=1 << 61)),
               dict(x_=0), dict(y=0), dict(x_=x.data_ptr() + 2), dict(mean=f.data_ptr()), dict(mean=f.data_ptr() + 1, rstd=f.data_ptr())):
        assert call(**kw) == qrm.QRM_E_INVALID and ctx.last_error(), kw
    assert lib.qrm_group_norm(h, None, x.data_ptr(), None, None, x.data_ptr(), None, None, None) == qrm.QRM_E_INVALID
    assert lib.qrm_group_norm(None, None, None, None, None, None, None, None, None) == qrm.QRM_E_INVALID
    assert call(change=dict(C=65538, groups=1)) == qrm.QRM_E_UNSUPPORTED
    assert call(change=dict(C=2047, groups=1, x_pixel=2047, y_pixel=2047)) == qrm.QRM_E_UNSUPPORTED  # 2047 pieces of four bytes
    d, p = qrm.group_norm_desc(**good), x.data_ptr()
    back = lambda dx, dg, mean=f.data_ptr(), dy=p: lib.qrm_group_norm_backward(h, C.byref(d), p, dy, None, None, mean, f.data_ptr(), dx, dg, None, None)
    assert back(None, None) == back(p, None, mean=None) == back(p, None, dy=None) == back(p, f.data_ptr() + 2) == qrm.QRM_E_INVALID
    assert back(None, f.data_ptr()) == 0
    torch.cuda.synchronize()


# ---------------------------------------------------------------- AdamW

SIZES = [1, 3, 0, 255, 256, 257, 1000, 4095, 4096, 4097, 10001, 40000]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


def make_plan(qrm, ctx, sizes, param, grad, copy, bits, seed, shift=0, warm=True):
    """Tensors `shift` elements into buffers of their own, with values and moments as in the middle of a training."""
    g = np.random.default_rng(seed)
    rows, refs, grads = [], [], []

    def put(value, dtype):
        buf = torch.full((value.size + shift + 8,), 9, dtype=dtype, device="cuda")
        t = buf[shift:shift + value.size]
        t.copy_(torch.from_numpy(value).to(dtype))
        t.buf = buf
        return t

    for i, n in enumerate(sizes):
        scale = 10.0 ** -(i % 5)
        p, gr = put(g.normal(0, 1, n).astype(np.float32), param), put((g.normal(0, 1, n) * scale).astype(np.float32), grad)
        m = (g.normal(0, 0.3, n) * scale * warm).astype(np.float32)
        v = ((g.random(n) * scale * warm) ** 2).astype(np.float32)
        t = dict(param=p, weight_decay=0.1 * (i % 3), lr_scale=1.0 + i % 2)
        if bits == 8:
            (cm, sm), (cv, sv) = ft.pack_moment(0, m), ft.pack_moment(1, v)
            t.update(m=put(cm, torch.int8), v=put(cv, torch.uint8), m_scale=torch.from_numpy(sm).cuda(), v_scale=torch.from_numpy(sv).cuda())
            m, v = ft.unpack_moment(0, cm, sm), ft.unpack_moment(1, cv, sv)
        else:
            t.update(m=put(m, torch.float32), v=put(v, torch.float32))
        if copy is not None:
            t["copy"] = put(np.zeros(n, np.float32), copy)
        rows.append(t)
        grads.append(gr)
        refs.append([f64(p), f64(gr), m.astype(np.float64), v.astype(np.float64)])
    return qrm.AdamW(ctx, rows, grad), rows, grads, refs


def check_step(rows, refs, step, param, copy, bits, scale=1.0, skip=(), shift=0):
    for i, (t, (p, g, m, v)) in enumerate(zip(rows, refs)):
        n = p.size
        if i in skip:
            assert np.array_equal(f64(t["param"]), p)
            if bits == 32:
                assert np.array_equal(f64(t["m"]), m) and np.array_equal(f64(t["v"]), v)
            continue
        rp, rm, rv = ft.adamw(p, g, m, v, step, weight_decay=t["weight_decay"], lr_scale=t["lr_scale"], grad_scale=scale, **HYPER)
        gs = np.abs(g * scale)
        slip_m = 6 * U * (HYPER["beta1"] * np.abs(m) + 0.1 * gs)                   # roundings of decoding, two products, a sum
        slip_v = 10 * U * rv
        move = np.abs(rp - p * (1 - HYPER["lr"] * t["lr_scale"] * t["weight_decay"]))
        # m's own slip goes through the quotient; eight roundings behind it
        rate = HYPER["lr"] * t["lr_scale"] / (1 - HYPER["beta1"] ** step)
        slip = rate * slip_m / (np.sqrt(rv / (1 - HYPER["beta2"] ** step)) + HYPER["eps"]) + 16 * U * move + 4 * U * np.abs(p)
        assert (np.abs(f64(t["param"]) - rp) <= slip + HALF[param] * (np.abs(rp) + slip) + TINY[param]).all()
        if copy is not None:
            assert (np.abs(f64(t["copy"]) - rp) <= slip + HALF[copy] * (np.abs(rp) + slip) + TINY[copy]).all()
        if bits == 32:
            assert (np.abs(f64(t["m"]) - rm) <= slip_m + 1e-45).all() and (np.abs(f64(t["v"]) - rv) <= slip_v + 1e-44).all()
        elif n:
            for which, code, got, value in ((0, t["m"], t["m_scale"], rm), (1, t["v"], t["v_scale"], rv)):
                rc, rs = ft.pack_moment(which, value)
                assert (np.abs(f64(got) - rs) <= 16 * U * rs).all()
                top = 127 if which == 0 else 255
                s = np.repeat(rs.astype(np.float64), 256)[:n]
                root = np.abs(value) if which == 0 else np.sqrt(value)
                y = top * np.sqrt(np.divide(root, s, out=np.zeros(n), where=s > 0))
                # codes are the nearest: another one only where the exact place lies between two, within what m's slip moves it
                c, r = np.abs(code.cpu().numpy().astype(int)), np.abs(rc.astype(int))
                near = np.abs(y - np.floor(y) - 0.5) <= 0.01 + 1e-4 * top
                assert ((c == r) | (near & (np.abs(c - r) <= 1))).all()
                assert (np.sign(code.cpu().numpy()) == np.sign(rc))[c == r].all()
        for key in ("param", "m", "v", "copy"):               # what lies before and behind the tensor is as it was
            if key in t:
                buf = t[key].buf
                assert bool((buf[:shift] == 9).all()) and bool((buf[shift + n:] == 9).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 4])
@pytest.mark.parametrize("param,grad,copy", [(torch.float32, torch.float32, None), (torch.float32, torch.bfloat16, torch.bfloat16),
                                             (torch.float32, torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16, None),
                                             (torch.float16, torch.float32, None)])
def test_adamw_step(ctx, qrm, param, grad, copy, bits, shift):
    for step in (1, 100):
        opt, rows, grads, refs = make_plan(qrm, ctx, SIZES, param, grad, copy, bits, seed=step, shift=shift, warm=step > 1)
        opt.qrm_adamw_step(grads, step, **HYPER)
        torch.cuda.synchronize()
        check_step(rows, refs, step, param, copy, bits, shift=shift)
        opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_tensors_without_gradient_and_a_scale_on_the_device(ctx, qrm, bits):
    opt, rows, grads, refs = make_plan(qrm, ctx, SIZES, torch.float32, torch.float32, None, bits, seed=3)
    skip = (0, 4, 10)
    before = [[t[k].clone() for k in ("m", "v")] for t in rows]
    opt.qrm_adamw_step([None if i in skip else g for i, g in enumerate(grads)], 5, d_grad_scale=torch.full((1,), 0.125, device="cuda"), **HYPER)
    torch.cuda.synchronize()
    check_step(rows, refs, 5, torch.float32, None, bits, scale=0.125, skip=skip)
    for i in skip:
        assert torch.equal(rows[i]["m"], before[i][0]) and torch.equal(rows[i]["v"], before[i][1])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [31, 32, 33, 447, 448, 449, 1000])
def test_adamw_many_tensors(ctx, qrm, count, bits):
    sizes = [(i * 37) % 301 for i in range(count)]
    opt, rows, grads, refs = make_plan(qrm, ctx, sizes, torch.float32, torch.bfloat16, torch.bfloat16, bits, seed=count)
    opt.qrm_adamw_step(grads, 9, **HYPER)
    torch.cuda.synchronize()
    check_step(rows, refs, 9, torch.float32, torch.bfloat16, bits)


def test_adamw_gradients_that_are_not_finite(ctx, qrm):
    for bits in (32, 8):
        opt, rows, grads, refs = make_plan(qrm, ctx, [700, 300], torch.float32, torch.float32, None, bits, seed=4)
        grads[0][300], grads[0][10] = float("nan"), float("inf")
        opt.qrm_adamw_step(grads, 3, **HYPER)
        p = f64(rows[0]["param"])
        assert np.isnan(p[[300, 10]]).all() and np.isfinite(np.delete(p, [300, 10])).all() and np.isfinite(f64(rows[1]["param"])).all()
        grads[0].zero_()
        opt.qrm_adamw_step(grads, 4, **HYPER)
        p = f64(rows[0]["param"])
        if bits == 32:
            assert np.isfinite(np.delete(p, [300, 10])).all()
        else:                                                # the first two blocks of 256 are spoilt, the third is not
            assert np.isnan(p[:512]).all() and np.isfinite(p[512:]).all()


def test_adamw_moments_that_fade(ctx, qrm):
    """Gradients of zero for good: moments fall to nothing and through the smallest numbers, parameters stay finite."""
    for bits in (32, 8):
        opt, rows, grads, _ = make_plan(qrm, ctx, [600], torch.float32, torch.float32, None, bits, seed=5)
        grads[0].zero_()
        for step in range(1, 1201):
            opt.qrm_adamw_step(grads, step, 1e-3, 0.9, 0.95, 1e-8)
        assert np.isfinite(f64(rows[0]["param"])).all()
        if bits == 8:
            out = torch.empty(600, device="cuda")
            for which in (0, 1):
                ctx.qrm_unpack_moment(which, rows[0]["mv"[which]], rows[0]["mv"[which] + "_scale"], 600, out)
                assert float(out.abs().max()) <= 1e-20


def test_adamw_tensor_of_more_than_2_31_elements(ctx, qrm):
    n = (1 << 31) + 300
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    parts = [slice(0, 1000), slice((1 << 31) - 500, n)]
    for s in parts:
        g[s].copy_(torch.randn(g[s].numel(), generator=torch.Generator().manual_seed(1)))
    opt = qrm.AdamW(ctx, [dict(param=p, m=m, v=v, m_scale=ms, v_scale=vs)], torch.bfloat16)
    opt.qrm_adamw_step([g], 1, 0.5, 0.9, 0.999, 1e-8)
    for s in parts:
        assert torch.equal(p[s].float(), -0.5 * torch.sign(g[s].float()))
    out = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    ctx.qrm_unpack_moment(0, m, ms, n, out)
    for s in parts:
        assert torch.allclose(out[s].float(), 0.1 * g[s].float(), rtol=0.0, atol=0.1 * 4.5 / 100)
    assert int((p != 0).sum()) == sum(int((g[s] != 0).sum()) for s in parts)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,shift", [(1, 0), (255, 0), (1024, 0), (1025, 1), (70000, 0), (70001, 3)])
def test_unpack_moment(ctx, n, shift, dtype):
    g = np.random.default_rng(n)
    scale = (10.0 ** g.uniform(-12, 2, -(-n // 256))).astype(np.float32)
    for which, code in ((0, g.integers(-127, 128, n).astype(np.int8)), (1, g.integers(0, 256, n).astype(np.uint8))):
        d = torch.full((n + 8,), 5, dtype=torch.int8 if which == 0 else torch.uint8, device="cuda")
        d[shift:shift + n] = torch.from_numpy(code).cuda()
        buf = torch.full((n + 8,), 5.0, dtype=dtype, device="cuda")
        ctx.qrm_unpack_moment(which, d[shift:shift + n], torch.from_numpy(scale).cuda(), n, buf[shift:shift + n])
        ref = ft.unpack_moment(which, code, scale)
        assert (np.abs(f64(buf[shift:shift + n]) - ref) <= (8 * U + HALF[dtype]) * np.abs(ref) + 2.0 ** -133).all()
        assert bool((buf[:shift] == 5).all()) and bool((buf[shift + n:] == 5).all())


def test_adamw_refusals(ctx, qrm):
    from paper_2509_02447_amd import binding as b
    lib, h = ctx._lib, ctx._h
    f = torch.zeros(1024, device="cuda")
    q = f.data_ptr()

    def create(desc=None, opt=True, **row):
        r = (b._AdamwTensor * 1)()
        for k, v in dict(dict(n=100, d_param=q, d_m=q, d_v=q, d_m_scale=q, d_v_scale=q, weight_decay=0.0, lr_scale=1.0), **row).items():
            setattr(r[0], k, v)
        d = b._AdamwDesc(*dict(dict(n_tensors=1, param_type=0, grad_type=0, copy_type=1, state_bits=32), **(desc or {})).values())
        out = C.c_void_p()
        st = lib.qrm_adamw_create(h, C.byref(d), r, C.byref(out) if opt else None)
        assert (st == 0) == bool(out.value)
        lib.qrm_adamw_destroy(out)
        return st

    assert create() == 0 and create(desc=dict(state_bits=8)) == 0 and create(n=0, d_param=None) == 0
    for desc in (dict(n_tensors=-1), dict(param_type=3), dict(grad_type=-1), dict(state_bits=16)):
        assert create(desc=desc) == qrm.QRM_E_INVALID, desc
    for row in (dict(n=-1), dict(d_param=None), dict(d_m=None), dict(d_v=q + 2), dict(d_copy=q + 1), dict(weight_decay=-1.0), dict(weight_decay=float("nan")),
                dict(lr_scale=float("inf"))):
        assert create(**row) == qrm.QRM_E_INVALID and ctx.last_error(), row
    assert create(desc=dict(state_bits=8), d_m_scale=None) == create(desc=dict(copy_type=0), d_copy=q) == qrm.QRM_E_INVALID
    assert create(desc=dict(param_type=1), d_copy=q) == create(opt=False) == qrm.QRM_E_INVALID
    assert create(n=1 << 44) == qrm.QRM_E_UNSUPPORTED
    lib.qrm_adamw_destroy(None)
    opt = qrm.AdamW(ctx, [dict(param=f[:100], m=f[100:200], v=f[200:300])], torch.float32)
    ptrs = (C.c_void_p * 1)(q)
    step = lambda n=1, lr=0.1, b1=0.9, b2=0.9, eps=1e-8, g=ptrs, o=opt._h, s=None: lib.qrm_adamw_step(h, o, g, n, lr, b1, b2, eps, s, None)
    assert step() == 0
    for kw in (dict(n=0), dict(lr=-1.0), dict(lr=float("nan")), dict(b1=1.0), dict(b2=-0.1), dict(b2=float("nan")), dict(eps=-1e-9), dict(eps=float("inf")),
               dict(g=None), dict(o=None), dict(s=q + 2), dict(g=(C.c_void_p * 1)(q + 1))):
        assert step(**kw) == qrm.QRM_E_INVALID, kw
    unpack = lambda which=0, codes=q, scales=q, n=10, typ=0, out=q: lib.qrm_unpack_moment(h, which, codes, scales, n, typ, out, None)
    assert unpack() == 0 and unpack(n=0, codes=None) == 0
    for kw in (dict(which=2), dict(codes=None), dict(scales=None), dict(out=None), dict(n=-1), dict(typ=2), dict(out=q + 1), dict(scales=q + 2)):
        assert unpack(**kw) == qrm.QRM_E_INVALID, kw
    with pytest.raises(AssertionError):
        opt.qrm_adamw_step([f[:99]], 1, 0.1)
    with pytest.raises(ValueError):
        qrm.AdamW(ctx, [dict(param=f[:9], m=f[:9], v=f[:9]), dict(param=f[:9].half(), m=f[:9], v=f[:9])], torch.float32)
    empty = qrm.AdamW(ctx, [], torch.float32)
    empty.qrm_adamw_step([], 1, 0.1)
    torch.cuda.synchronize()


# ---------------------------------------------------------------- message loss

CODES = {2: (3, 1, 0x7), 3: (7, 3, 0xB), 4: (12, 8, 0x13), 5: (20, 10, 0x25), 6: (21, 5, 0x43), 7: (18, 4, 0x89), 8: (12, 8, 0x11D)}


def check_loss(ctx, n, m, bits, t, weight, target, logits, symbols=True, grad=True):
    d = torch.from_numpy(logits).cuda()
    loss = torch.full((1,), np.nan, device="cuda")
    dz = torch.full((n, bits), np.nan, device="cuda") if grad else None
    be, se = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    ctx.qrm_message_loss(d, torch.from_numpy(target).cuda(), 1 if target.ndim == 1 else n, n, bits, weight, loss, dz, be, se if symbols else None)
    torch.cuda.synchronize()
    rl, rg, rb, rs = ft.message_loss(logits, target, m, t, weight)
    assert np.array_equal(be.cpu().numpy(), rb) and (not symbols or np.array_equal(se.cpu().numpy(), rs))
    # E is a sum of at most `bits` numbers of up to 1, each within m + 4 roundings; its excess over t is squared
    one = np.broadcast_to(target != 0, logits.shape)
    x = np.where(one, logits, -logits).astype(np.float64)
    bce = np.maximum(-x, 0) + np.log1p(np.exp(-np.abs(x)))
    right = np.exp(-bce.reshape(n, bits // m, m).sum(axis=2))
    slip_right = right * (8 + bce.reshape(n, bits // m, m).sum(axis=2) * 8) * U
    slip_e = slip_right.sum(axis=1) + (bits // m) * 8 * U
    over = np.maximum((1 - right).sum(axis=1) - t, 0)
    assert abs(float(loss[0]) - rl) <= 16 * U * (rl + 1e-30) + weight / n * (slip_e * (2 * over + slip_e)).sum() + 16 * U * bce.sum() / (n * bits)
    if grad:
        miss = ft._sigmoid(-x)
        slip = 2 * weight / n * (over[:, None] * slip_right + slip_e[:, None] * right)
        tol = 24 * U * np.abs(rg) + miss * np.repeat(slip, m, axis=1) + 2.0 ** -149
        assert (np.abs(f64(dz) - rg) <= tol).all()


@pytest.mark.parametrize("m", sorted(CODES))
@pytest.mark.parametrize("n", [1, 3, 17, 256, 257, 5000])
def test_message_loss(qrm, m, n):
    length, k, poly = CODES[m]
    ctx = qrm.Context(rs=dict(m=m, prim_poly=poly, n=length, k=k, fcr=1))
    g = np.random.default_rng(n + m)
    bits, t = m * length, (length - k) // 2
    for shared, weight in ((False, 1.0), (True, 0.3), (False, 0.0)):
        target = g.integers(0, 2, (bits,) if shared else (n, bits)).astype(np.uint8) * (255 if shared else 1)
        logits = (g.normal(0, 2, (n, bits)) + (np.broadcast_to(target, (n, bits)).astype(float).clip(0, 1) * 2 - 1)).astype(np.float32)
        check_loss(ctx, n, m, bits, t, weight, target, logits, grad=weight != 0.3 or n != 17)
    ctx.close()


@pytest.mark.parametrize("m,length,k,poly", [(8, 255, 239, 0x11D), (8, 65, 49, 0x11D), (7, 127, 111, 0x89)])
def test_message_loss_long_words(qrm, m, length, k, poly):
    ctx = qrm.Context(rs=dict(m=m, prim_poly=poly, n=length, k=k, fcr=1))
    g = np.random.default_rng(1)
    for n in (1, 40, 130):
        target = g.integers(0, 2, (n, m * length)).astype(np.uint8)
        logits = (g.normal(0, 2, target.shape) + (target * 6.0 - 3.0)).astype(np.float32)
        check_loss(ctx, n, m, m * length, (length - k) // 2, 1.0, target, logits)
    ctx.close()


def test_message_loss_without_a_code(qrm):
    import synth
    cfg = synth.CONFIGS["C1"]
    ctx = qrm.Context(weights=synth.config_weights(cfg))
    g = np.random.default_rng(2)
    for n, bits in ((1, 1), (5, 33), (300, 60), (4, 2040)):
        target = g.integers(0, 2, (n, bits)).astype(np.uint8)
        check_loss(ctx, n, 1, bits, 0, 0.0, target, g.normal(0, 2, target.shape).astype(np.float32), symbols=False)
    z = torch.zeros((2, 8), device="cuda")
    for kw in (dict(w=1.0), dict(se=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(qrm.QrmError):
            ctx.qrm_message_loss(z, z.to(torch.uint8), 2, 2, 8, kw.get("w", 0.0), torch.zeros(1, device="cuda"), None, None, kw.get("se"))
    ctx.close()


@pytest.mark.parametrize("n", [2, 900])
def test_message_loss_logits_that_are_far_off_or_not_finite(ctx, n):
    g = np.random.default_rng(6)
    target = g.integers(0, 2, (n, 48)).astype(np.uint8)
    logits = g.normal(0, 2, (n, 48)).astype(np.float32)
    far = logits.copy()
    far[0, :4] = [1e4, -1e4, 3e38, -3e38]
    far[1, 8:12] = [90.0, -90.0, 110.0, -110.0]
    check_loss(ctx, n, 4, 48, 2, 1.0, target, far)
    bad = logits.copy()
    bad[1, 5] = np.nan
    dz = torch.empty((n, 48), device="cuda")
    loss = torch.empty(1, device="cuda")
    ctx.qrm_message_loss(torch.from_numpy(bad).cuda(), torch.from_numpy(target).cuda(), n, n, 48, 1.0, loss, dz)
    rows = torch.isnan(dz).any(dim=1).cpu()
    assert bool(torch.isnan(loss).all()) and bool(rows[1]) and int(rows.sum()) == 1
    sure = np.where(target != 0, np.inf, -np.inf).astype(np.float32)
    ctx.qrm_message_loss(torch.from_numpy(sure).cuda(), torch.from_numpy(target).cuda(), n, n, 48, 1.0, loss, dz)
    assert float(loss[0]) == 0.0 and not bool(dz.any())


def test_message_loss_no_images_and_refusals(ctx, qrm):
    loss = torch.full((1,), 5.0, device="cuda")
    z, target = torch.zeros((0, 48), device="cuda"), torch.zeros((1, 48), dtype=torch.uint8, device="cuda")
    ctx.qrm_message_loss(z, target, 1, 0, 48, 1.0, loss, z)
    assert float(loss[0]) == 0.0
    lib, h, q, p = ctx._lib, ctx._h, torch.zeros(96, device="cuda"), loss.data_ptr()
    call = lambda logits=q.data_ptr(), tgt=target.data_ptr(), rows=1, n=2, bits=48, w=1.0, out=p, grad=None, be=None: lib.qrm_message_loss(
        h, logits, tgt, rows, n, bits, w, out, grad, be, None, None)
    assert call() == 0
    for kw in (dict(logits=None), dict(tgt=None), dict(rows=0), dict(rows=3), dict(n=-1), dict(bits=47), dict(bits=0), dict(w=-0.1), dict(w=float("nan")),
               dict(w=float("inf")), dict(out=None), dict(out=p + 2), dict(grad=q.data_ptr() + 1), dict(be=p + 2)):
        assert call(**kw) == qrm.QRM_E_INVALID and ctx.last_error(), kw
    assert call(n=(1 << 31) // 64, rows=1) == qrm.QRM_E_UNSUPPORTED
    torch.cuda.synchronize()


def test_message_loss_same_bits_again(ctx):
    g = np.random.default_rng(9)
    for n in (4, 20000):
        z = torch.from_numpy(g.normal(0, 2, (n, 48)).astype(np.float32)).cuda()
        target = torch.from_numpy(g.integers(0, 2, (n, 48)).astype(np.uint8)).cuda()
        outs = []
        for _ in range(5):
            loss, dz = torch.empty(1, device="cuda"), torch.empty((n, 48), device="cuda")
            ctx.qrm_message_loss(z, target, n, n, 48, 1.0, loss, dz)
            outs.append((loss, dz))
        assert all(torch.equal(a, b) for o in outs for a, b in zip(o, outs[0]))


def test_a_recorded_step_gives_the_eager_step_at_every_replay(ctx, qrm):
    """Norm, its backward pass, the loss and AdamW in one graph, replayed with eager work of the same context in between."""
    n, p, c, groups, bits = 3, 9000, 64, 8, 48
    g = torch.Generator().manual_seed(21)
    x, dy = (torch.randn((n, p, c), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    logits, target = torch.randn((6000, bits), generator=g).cuda(), torch.randint(0, 2, (bits,), generator=g, dtype=torch.uint8).cuda()
    grad = torch.randn(5000, generator=g).cuda()
    d = qrm.group_norm_desc(n, p, c, groups, x.dtype, "silu")

    def state():
        o = dict(y=torch.empty_like(x), mean=torch.empty((n, groups), device="cuda"), rstd=torch.empty((n, groups), device="cuda"), dx=torch.empty_like(x),
                 dgamma=torch.empty(c, device="cuda"), dbeta=torch.empty(c, device="cuda"), loss=torch.empty(1, device="cuda"), dz=torch.empty_like(logits),
                 p=torch.ones(5000, device="cuda"), m=torch.zeros(5000, dtype=torch.int8, device="cuda"), v=torch.zeros(5000, dtype=torch.uint8, device="cuda"),
                 ms=torch.zeros(20, device="cuda"), vs=torch.zeros(20, device="cuda"))
        return o, qrm.AdamW(ctx, [dict(param=o["p"], m=o["m"], v=o["v"], m_scale=o["ms"], v_scale=o["vs"])], torch.float32)

    def step(o, opt):
        ctx.qrm_group_norm(d, x, None, None, o["y"], o["mean"], o["rstd"])
        ctx.qrm_group_norm_backward(d, x, dy, None, None, o["mean"], o["rstd"], o["dx"], o["dgamma"], o["dbeta"])
        ctx.qrm_message_loss(logits, target, 1, 6000, bits, 1.0, o["loss"], o["dz"])
        opt.qrm_adamw_step([grad], 3, 1e-3)

    (eager, eager_opt), (seen, seen_opt) = state(), state()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):                          # the stream's workspace is there before the recording
        step(seen, seen_opt)
    step(eager, eager_opt)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(seen, seen_opt)
    for _ in range(4):
        for k in ("y", "mean", "dx", "dgamma", "loss", "dz"):
            seen[k].fill_(5)
        with torch.cuda.stream(stream):
            graph.replay()
        step(eager, eager_opt)
        torch.cuda.synchronize()
        for k in eager:
            assert torch.equal(eager[k], seen[k]), k
        logits.mul_(0.9), x.mul_(1.25)                       # other inputs at the same addresses
        torch.cuda.synchronize()
    ctx.qrm_release_stream(stream)
