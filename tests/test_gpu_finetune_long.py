"""Group norms of so many images that a thread walks down thousands of pixels: what it adds up stays within the bounds that short sums have.

The inputs are those whose roundings all go one way: a gradient that is the same at every pixel, values whose squares are.  u = 2^-24.  A thread adds 48
pixels, the sums of up to 43 such runs, a few rows' sums; those are added in 64 bits: within 128 u of the sum of the magnitudes (equal numbers added one after
the other in 32 bits are off by 240 u after 1024 of them and by 1000 u after 4096)."""
import numpy as np
import pytest
import torch

from oracle import finetune as ft

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
IMAGES = 257                                                 # (one workgroup to a tile of an image, on 256 compute units)


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(qrm):
    c = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    yield c
    c.close()


def maps(pixels, channels, pitch):
    return torch.empty((IMAGES, pixels, pitch), device="cuda")[:, :, :channels]


# channels, their distance, groups, pixels: single channels, four at once; 4096 pixels a thread
@pytest.mark.parametrize("c,pitch,groups,p", [(31, 31, 31, 32768), (32, 32, 4, 131072)])
def test_gradients_that_are_the_same_everywhere(ctx, qrm, c, pitch, groups, p):
    x, dy = maps(p, c, pitch), maps(p, c, pitch)
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(c))
    dy.fill_(0.1)
    gradient = float(dy[0, 0, 0])
    rows = x.view(IMAGES, p, groups, -1)
    mean = torch.stack([r.double().mean(dim=(0, 2)) for r in rows]).float()
    rstd = torch.ones_like(mean)
    dgamma, dbeta = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    first = x[0].double().cpu().numpy()[None]
    d = qrm.group_norm_desc(IMAGES, p, c, groups, torch.float32, "none", 1e-6, pitch, p * pitch, pitch, p * pitch)
    ctx.qrm_group_norm_backward(d, x, dy, None, None, mean, rstd, dy, dgamma, dbeta)
    want = IMAGES * p * gradient
    assert (np.abs(dbeta.double().cpu().numpy() - want) <= 128 * U * want).all()
    # dx of the first image: gradient, its mean and what h takes of it, each mean within 128 u of its magnitudes; a dozen roundings
    m = mean[:1].double().cpu().numpy()
    rdx = ft.group_norm_backward(first, np.full_like(first, gradient), None, None, m, np.ones_like(m), groups, "none")[0]
    h = np.abs(first - np.repeat(m, c // groups, 1)[:, None])
    share = np.repeat(h.reshape(1, p, groups, -1).mean(axis=(1, 3)), c // groups, 1)[:, None]
    tol = 140 * U * gradient * (2 + h * share)
    err = np.abs(dy[:1].double().cpu().numpy() - rdx)
    assert (err <= tol).all(), f"off by {(err / tol).max()} of what is allowed"


def test_values_whose_squares_are_the_same_everywhere(ctx, qrm):
    """Squares about the mean: sets of eight pixels are joined one after the other, 256 at most to a thread; with the eight, the rows of a
    workgroup and the chunks of an image under 300 roundings of the sum, half of that in its root."""
    p, c = 262144, 31
    x = maps(p, c, c)
    x[:] = torch.where(torch.arange(p, device="cuda") // 8 % 2 == 0, 0.9, -0.9).view(1, p, 1)
    value = float(x[0, 0, 0])
    mean, rstd = torch.empty((IMAGES, c), device="cuda"), torch.empty((IMAGES, c), device="cuda")
    ctx.qrm_group_norm(qrm.group_norm_desc(IMAGES, p, c, c, torch.float32), x, None, None, x, mean, rstd)
    want = 1.0 / np.sqrt(value * value + float(np.float32(1e-6)))
    assert float(mean.abs().max()) <= 150 * U * value
    assert float((rstd.double() / want - 1).abs().max()) <= 150 * U
