"""Which tensors the binding takes for a map [N,P,C] with given strides (no GPU): those whose elements lie where the map's do, and no others."""
import itertools
import random

import pytest
import torch

from paper_2509_02447_amd import binding


def test_maps_as_callers_write_them():
    lies = binding._lies
    t = torch.empty(2, 10, 8)
    for v in (t, t.view(2, 2, 5, 8), t.view(20, 8), t.view(-1), t.view(2, 80), t.view(1, 2, 10, 8)):
        assert lies(v, 2, 10, 8, 8, 80)
    wide = torch.empty(2, 10, 12)
    part = wide[:, :, :8]
    for v in (part, wide, part.unflatten(1, (2, 5)), wide.view(-1)):
        assert lies(v, 2, 10, 8, 12, 120)                    # a part of the channels, or the buffer that it is a part of
        assert not lies(v, 2, 10, 8, 8, 80) or v.dim() == 1
    assert lies(t, 1, 10, 8, 8, 80) and lies(wide, 1, 10, 8, 12, 120)      # more images than asked for
    for n, p, c in ((2, 9, 8), (3, 10, 8), (2, 10, 9), (2, 20, 8)):
        assert not lies(t, n, p, c, c, p * c)
    assert not lies(t.transpose(0, 1), 2, 10, 8, 8, 80) and not lies(t.transpose(1, 2), 2, 8, 10, 10, 80)
    assert not lies(t[:, ::2], 2, 5, 8, 8, 40) and lies(t[:, ::2], 2, 5, 8, 16, 80)
    assert not lies(t.view(-1)[:159], 2, 10, 8, 8, 80)
    assert lies(torch.empty(0, 10, 8), 0, 10, 8, 8, 80)


@pytest.mark.parametrize("seed", range(4))
def test_what_is_taken_lies_as_the_map_does(seed):
    """Tensors of random shapes and strides beside random maps: places of their elements, spelt out.  A tensor of just the map's pixels that
    lies right is taken, too."""
    r, taken = random.Random(seed), 0
    places = torch.arange(4000)
    for _ in range(3000):
        n, p, c = r.randint(1, 3), r.randint(1, 6), r.randint(1, 3)
        pixel = c + r.choice([0, 0, 1, 2])
        image = p * pixel + r.choice([0, 0, 3])
        shape = [r.randint(1, 6) for _ in range(r.randint(2, 4))]
        kind = r.random()
        if kind < 0.2:
            shape = [n * p, c]
        elif kind < 0.6:
            shape = [n, 2, 3, c] if p == 6 and kind < 0.4 else [n, p, c + r.choice([0, 0, 1])]
        usual = {2: [pixel, 1], 3: [image, pixel, 1], 4: [image, 3 * pixel, pixel, 1]}[len(shape)]
        some = [r.choice([pixel, image, p * pixel, 3 * pixel, c, 1]) for _ in shape[1:]] + [1]
        stride = r.choice([usual, usual, some, list(torch.empty(shape).stride())])
        t = places.as_strided(shape, stride)
        took = binding._lies(t, n, p, c, pixel, image)
        taken += took
        if shape[-1] < c:
            assert not took or (t.is_contiguous() and t.numel() == n * p * c and pixel == c and (n == 1 or image == p * c))
            continue
        mine = t[..., :c].reshape(-1, c)
        want = torch.tensor([[i * image + k * pixel + j for j in range(c)] for i, k in itertools.product(range(n), range(p))])
        right = mine.shape[0] >= n * p and torch.equal(mine[:n * p], want)
        if took:
            assert right or torch.equal(t.reshape(-1), want.reshape(-1)), (shape, stride, n, p, c, pixel, image)
        elif mine.shape[0] == n * p:
            assert not right, (shape, stride, n, p, c, pixel, image)
    assert taken > 300


def test_a_descriptor_that_is_changed_says_so():
    d = binding.group_norm_desc(2, 10, 8, 4, torch.bfloat16, "silu")
    assert d.maps() == (torch.bfloat16, (2, 10, 8), (80, 8, 1), (80, 8, 1), 8)
    d.x_pixel, d.y_image, d.N = 12, 99, 3
    assert d.maps() == (torch.bfloat16, (3, 10, 8), (120, 12, 1), (99, 8, 1), 12)
    d.type = 7
    assert d.maps()[0] is None and d.type == 7 and d.P == 10
    d.groups, d.type = 2, binding.QRM_F32
    assert d.maps() == (torch.float32, (3, 10, 8), (120, 12, 1), (99, 8, 1), 6)
