"""How wide a group of a group norm may be: D channels that are D / gcd(D, V) pieces, V elements read at once, up to 1024."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(qrm):
    c = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("c,groups", [(8200, 4), (8192, 4), (8216, 8), (8184, 8), (1025, 1), (1023, 1), (2050, 1), (2046, 1), (2052, 1), (4100, 1), (4096, 1), (8192, 1),
                                      (8196, 2), (6150, 3)])
def test_wide_groups_by_the_rule(ctx, qrm, c, groups, dtype):
    widest = 8 if dtype is torch.bfloat16 else 4
    at_once = math.gcd(c, widest)                            # dense maps on 16-byte boundaries
    d = c // groups
    x = torch.randn((2, 3, c), generator=torch.Generator().manual_seed(c)).to(dtype).cuda()
    y, stats = torch.empty_like(x), torch.empty((2, groups), device="cuda")
    call = lambda: ctx.qrm_group_norm(qrm.group_norm_desc(2, 3, c, groups, dtype), x, None, None, y, stats, stats.clone())
    if d // math.gcd(d, at_once) > 1024:
        with pytest.raises(qrm.QrmError, match="1024 pieces") as e:
            call()
        assert e.value.status == qrm.QRM_E_UNSUPPORTED
    else:
        call()
        want = x.double().view(2, 3, groups, d).mean(dim=(1, 3))
        assert float((stats.double() - want).abs().max()) <= 1e-5
