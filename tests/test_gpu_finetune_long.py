"""Group norms of so many images that a thread walks down thousands of pixels: what it adds up stays within the bounds that short sums have.

The inputs are those whose roundings all go one way: values whose squares are the same.  u = 2^-24."""
import numpy as np
import pytest
import torch

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
