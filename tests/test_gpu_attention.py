"""Attention and its backward pass on the GPU, through the C ABI, against the 64-bit oracle (oracle/attention.py).

Tolerances come from the number formats: u = 2^-24 is half a unit in the last place of 32 bits, `half` that of the type.  A score is a sum of D products
(D + 8 roundings, with the scale, the exponent's argument and the exponential), sums over rows follow each other (a rounding a row, and a few for parts that are
joined), probabilities and score gradients of 16-bit types are rounded once more (half), results once (half).
"""
import numpy as np
import pytest
import torch

from oracle import attention as at

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}
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


def rows_of(shape, dtype, layout="rows", gap=0, shift=0, fill=0.0):
    """(buffer, view [N,L,heads,D]) with `gap` elements behind every row (layout "rows") or head ("heads"), `shift` elements in."""
    n, l, h, d = shape
    if layout == "heads":
        strides = (h * l * (d + gap), d + gap, l * (d + gap), 1)
    else:
        strides = (l * h * (d + gap), h * (d + gap), d + gap, 1)
    size = 1 + sum((s - 1) * st for s, st in zip(shape, strides) if s > 0) if min(shape) > 0 else 0
    buf = torch.full((shift + size + 64,), fill, dtype=dtype, device="cuda")
    return buf, buf.as_strided(shape, strides, shift)


def desc_of(qrm, q, k, v, o, causal, scale):
    lie = lambda t: (t.stride(1), t.stride(2), t.stride(0))
    return qrm.attention_desc(q.shape[0], q.shape[1], k.shape[1], q.shape[2], k.shape[2], q.shape[3], q.dtype, causal, scale, lie(q), lie(k), lie(v), lie(o))


def lens_tensor(lens):
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


class Case:
    def __init__(self, qrm, n, lq, lk, heads, kv, d, dtype, causal=False, q_len=None, k_len=None, layout="rows", gap=0, shift=0, seed=0, spread=1.4, scale=None, rest=np.nan):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.causal, self.q_len, self.k_len = dtype, causal, q_len, k_len
        self.scale = float(np.float32(d ** -0.5 if scale is None else scale))
        normal = lambda shape, std: torch.randn(shape, generator=g) * std
        self.bufs = {}

        def place(name, shape, value=None, fill=0.0):
            self.bufs[name], view = rows_of(shape, dtype, layout, gap, shift, fill)
            if value is not None:
                view.copy_(value.to(dtype))
            return view

        self.q = place("q", (n, lq, heads, d), normal((n, lq, heads, d), spread))
        self.k = place("k", (n, lk, kv, d), normal((n, lk, kv, d), 1.0) + normal((1, 1, kv, d), 0.4))
        self.v = place("v", (n, lk, kv, d), normal((n, lk, kv, d), 1.0) + normal((1, 1, kv, d), 0.7))
        self.do = place("do", (n, lq, heads, d), normal((n, lq, heads, d), 0.05))
        self.o = place("o", (n, lq, heads, d), None, 7.0)
        self.dq, self.dk, self.dv = place("dq", self.q.shape, None, 7.0), place("dk", self.k.shape, None, 7.0), place("dv", self.v.shape, None, 7.0)
        # rows that are not there hold what must not matter
        for lens, tensors in ((q_len, (self.q, self.do)), (k_len, (self.k, self.v))):
            for i, m in enumerate(lens or []):
                for t in tensors:
                    t[i, max(m, 0):] = rest
        self.lse = torch.full((n, heads, lq), 7.0, device="cuda")
        self.desc = desc_of(qrm, self.q, self.k, self.v, self.o, causal, self.scale)
        self.lens = lens_tensor(q_len), lens_tensor(k_len)
        self.args = tuple(np.nan_to_num(f64(t), nan=0.0) for t in (self.q, self.k, self.v))

    def forward(self, ctx, lse=True):
        ctx.qrm_attention(self.desc, self.q, self.k, self.v, self.o, self.lse if lse else None, *self.lens)

    def backward(self, ctx):
        ctx.qrm_attention_backward(self.desc, self.q, self.k, self.v, self.o, self.do, self.lse, self.dq, self.dk, self.dv, *self.lens)

    def score_off(self):
        return (self.q.shape[3] + 8) * U

    def check_forward(self):
        q, k, v = self.args
        o, lse, weight = at.attention(q, k, v, self.scale, self.causal, self.q_len, self.k_len)
        d, lk, half = q.shape[3], k.shape[1], HALF[self.dtype]
        big = self.scale * np.abs(q).max(initial=0) * np.abs(k).max(initial=0) * d  # no sum of |q| |k| is larger
        scores = self.score_off() * (1.0 + 2.0 * big)
        got = f64(self.lse)
        assert np.array_equal(np.isneginf(got), np.isneginf(lse)), "rows that see nothing"
        fine = np.isfinite(lse)
        assert (np.abs(got[fine] - lse[fine]) <= scores + (lk + 16) * U + 4 * U * np.abs(lse[fine])).all()
        rounded = 0.0 if self.dtype == torch.float32 else half
        tol = (rounded + 2 * scores + (2 * lk + 32) * U) * weight * 1.01 + half * np.abs(o) + TINY[self.dtype]
        if self.dtype == torch.float16:                                   # probabilities below 2^-14 of the largest are rounded to 2^-25 of it
            tol += lk * 2.0 ** -25 * np.abs(v).max(initial=0)
        err = np.abs(f64(self.o) - o)
        assert (err <= tol).all(), f"off by {(err / tol).max()} of what is allowed"

    def check_backward(self, outputs=("dq", "dk", "dv")):
        q, k, v = self.args
        d, half = q.shape[3], HALF[self.dtype]
        rounded = 0.0 if self.dtype == torch.float32 else half
        rows = k.shape[1] + q.shape[1] * (q.shape[2] // k.shape[2])
        do, o = np.nan_to_num(f64(self.do), nan=0.0), f64(self.o)
        grads, off = at.attention_backward(q, k, v, o, do, f64(self.lse), self.scale, self.causal, self.q_len, self.k_len, self.score_off(), (d + 4) * U, rounded, (rows + 16) * U)
        for name, want, far in zip(("dq", "dk", "dv"), grads, off):
            if name not in outputs:
                continue
            # (f16: what is under 2^-29 of a row's largest may be lost in a sum: `rows` of them)
            tol = far * 1.01 + half * np.abs(want) + TINY[self.dtype] + (rows * 2.0 ** -24 * far.max(initial=0) if self.dtype == torch.float16 else 0.0)
            err = np.abs(f64(getattr(self, name)) - want)
            assert (err <= tol).all(), f"{name} off by {(err / tol).max()} of what is allowed"

    def check_gaps(self, names):
        for name in names:
            getattr(self, name).fill_(7.0)
            assert bool((self.bufs[name] == 7.0).all()), f"{name}: something beside its rows was written"


def check(ctx, qrm, *args, **kw):
    c = Case(qrm, *args, **kw)
    c.forward(ctx)
    torch.cuda.synchronize()
    c.check_forward()
    c.backward(ctx)
    torch.cuda.synchronize()
    c.check_backward()
    c.check_gaps(("o", "dq", "dk", "dv"))
    return c


# single rows, one more and less than a wavefront's columns, than a workgroup's and than a tile; every width class and both sides of its borders
SHAPES = [(1, 1, 1, 1, 1, 8), (1, 1, 1, 1, 1, 1), (2, 31, 33, 2, 2, 64), (1, 33, 31, 1, 1, 72), (2, 65, 64, 4, 2, 40), (1, 129, 127, 3, 1, 128), (3, 17, 200, 2, 1, 16),
          (1, 200, 17, 6, 3, 96), (2, 64, 65, 1, 1, 136), (1, 130, 100, 2, 2, 256), (1, 70, 90, 1, 1, 264), (2, 33, 100, 1, 1, 512), (1, 128, 96, 2, 1, 512), (1, 300, 515, 1, 1, 48)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(ctx, qrm, shape, dtype):
    for causal in (False, True):
        check(ctx, qrm, *shape, dtype, causal=causal, seed=sum(shape))


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("layout,gap,shift", [("rows", 0, 0), ("heads", 0, 0), ("rows", 8, 8), ("heads", 16, 0), ("rows", 3, 0), ("heads", 1, 1), ("rows", 0, 1), ("heads", 0, 4)])
def test_layouts_strides_and_alignment(ctx, qrm, layout, gap, shift, dtype):
    check(ctx, qrm, 2, 45, 70, 4, 2, 32, dtype, causal=True, layout=layout, gap=gap, shift=shift, seed=gap + shift, q_len=[45, 20], k_len=[61, 70])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("d", [1, 3, 7, 13, 33, 61, 100, 127, 130, 255, 301, 511])
def test_odd_row_lengths(ctx, qrm, d, dtype):
    check(ctx, qrm, 1, 37, 53, 2, 1, d, dtype, seed=d)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("d", [32, 40, 96, 104, 128, 192, 200, 256, 264])
def test_row_lengths_on_both_sides_of_a_kernels(ctx, qrm, d, dtype):
    check(ctx, qrm, 1, 140, 150, 2, 1, d, dtype, causal=True, seed=d)


@pytest.mark.parametrize("n,kv", [(1, 2), (3, 1), (1, 4), (5, 1), (2, 3), (7, 1), (4, 2), (3, 3), (1, 16), (17, 1)])
def test_numbers_of_key_heads(ctx, qrm, n, kv):
    """They are dealt to the dies in ways of their own below eight, at eight and above."""
    check(ctx, qrm, n, 300, 260, 2 * kv, kv, 64, torch.bfloat16, causal=True, seed=n + kv)
    check(ctx, qrm, n, 2, 700, 2 * kv, kv, 64, torch.float32, seed=n + kv)


def test_rows_and_images_more_than_2_31_elements_apart(ctx, qrm):
    """Keys 2^21 elements apart, and a second image 2^31 behind the first: offsets of 32 bits would meet other rows."""
    d, lk, lq = 64, 1100, 70
    g = torch.Generator().manual_seed(0)
    apart, image = 1 << 21, (1 << 31) + (1 << 28)
    wide = torch.zeros(image + lk * apart, dtype=torch.bfloat16, device="cuda")
    c = Case(qrm, 2, lq, lk, 1, 1, d, torch.bfloat16, causal=True, seed=6)
    k = wide.as_strided((2, lk, 1, d), (image, apart, d, 1), 0)
    v = wide.as_strided((2, lk, 1, d), (image, apart, d, 1), 4096)
    dk, dv = wide.as_strided((2, lk, 1, d), (image, apart, d, 1), 8192), wide.as_strided((2, lk, 1, d), (image, apart, d, 1), 12288)
    k.copy_(c.k), v.copy_(c.v)
    c.k, c.v, c.dk, c.dv = k, v, dk, dv
    c.desc = desc_of(qrm, c.q, k, v, c.o, True, c.scale)
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [64, 200])
def test_lengths_and_rows_that_see_nothing(ctx, qrm, causal, d, dtype):
    # none, one, tile borders, all, less than none and more than all; queries longer than their keys see nothing in the beginning where causal
    q_len, k_len = [0, 100, 1, 64, 100, 77, -3, 1000], [50, 0, 1, 64, 130, 31, 20, 2000]
    check(ctx, qrm, 8, 100, 130, 4, 2, d, dtype, causal=causal, q_len=q_len, k_len=k_len, seed=5)
    c = Case(qrm, 8, 100, 130, 4, 2, d, dtype, causal=causal, q_len=q_len, k_len=k_len, seed=5)
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    assert bool((c.o[0] == 0).all()) and bool((c.o[1] == 0).all()) and bool((c.dq[1] == 0).all()) and bool((c.dk[4, 130:] == 0).all())
    assert bool((c.dv[2, 1:] == 0).all()) and bool((c.dq[2, 1:] == 0).all()) and bool(torch.isfinite(c.dk.float()).all())
    if causal:
        assert bool((c.o[5, :46] == 0).all()) and bool(torch.isneginf(c.lse[5, :, :46]).all()) and bool(torch.isfinite(c.lse[5, :, 46:77]).all())


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("group", [1, 3, 8, 40])
@pytest.mark.parametrize("lq", [1, 2, 5])
def test_single_tokens_over_long_rows(ctx, qrm, lq, group, dtype):
    for d in (64, 128, 320):
        check(ctx, qrm, 3, lq, 3001, 2 * group, 2, d, dtype, causal=lq > 1, k_len=[3001, 1, 1500], seed=group)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,lq,lk,heads,kv,d,causal", [(1, 1024, 1024, 1, 1, 512, False), (1, 2257, 2257, 2, 1, 60, True), (2, 1500, 77, 4, 4, 40, False), (1, 300, 5000, 1, 1, 128, True),
                                                     (1, 5000, 300, 2, 2, 128, True), (1, 40, 40000, 1, 1, 64, False)])
def test_long_rows(ctx, qrm, n, lq, lk, heads, kv, d, causal, dtype):
    check(ctx, qrm, n, lq, lk, heads, kv, d, dtype, causal=causal, seed=lq)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_scores_far_apart(ctx, qrm, dtype):
    # one key has nearly all weight, or none: differences of hundreds
    check(ctx, qrm, 1, 100, 150, 2, 2, 64, dtype, seed=1, spread=25.0)
    check(ctx, qrm, 1, 100, 150, 2, 2, 64, dtype, seed=2, scale=1e-4)


def test_small_gradients_in_f16(ctx, qrm):
    """Score gradients of 2^-30 and less are under the type's smallest number; their products with rows of 2^10 are not."""
    c = Case(qrm, 1, 600, 700, 2, 1, 64, torch.float16, seed=3)
    c.do.mul_(2.0 ** -8)
    c.k.mul_(2.0 ** 3)
    c.q.mul_(2.0 ** -3)
    c.args = tuple(f64(t) for t in (c.q, c.k, c.v))
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    c.check_forward()
    c.check_backward()
    assert float(c.dq.float().abs().mean()) > 0


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_many_keys_of_little_weight(ctx, qrm, dtype):
    """2^17 keys of exp(-18) each beside one of weight 1: together 0.2 %, each less than half of f16's smallest number.  The weights' rounding (f16: to steps of
    2^-24 / 2^11 at least), 2^17 / 8 additions to a lane's sum, the result's rounding; and the products' sums: an instruction adds the products of two rows (f32) or more
    to what there is, so 2^17 / 2 roundings of equal summands, which all go the same way."""
    lq, lk, heads, d = 1024, 1 << 17, 64, 32
    q = torch.zeros((1, lq, heads, d), dtype=dtype, device="cuda")
    k, v = (torch.zeros((1, lk, 1, d), dtype=dtype, device="cuda") for _ in range(2))
    q[..., 0], k[..., 0], v[...] = 4.0, -4.5, 1.0
    k[0, 77], v[0, 77] = 0.0, 0.0
    o = torch.empty_like(q)
    ctx.qrm_attention(desc_of(qrm, q, k, v, o, False, 1.0), q, k, v, o, None, None, None, 0)
    p = float(np.exp(-18.0))
    weight = (lk - 1) * p
    want = weight / (1.0 + weight)
    half = HALF[dtype]
    tolerance = (2 * half + lk / 8 * U + lk / 2 * U + 64 * U + (2.0 ** -36 / p if dtype == torch.float16 else 0.0)) * 1.01
    off = float((o.double() / want - 1.0).abs().max())
    assert off <= tolerance, (off, tolerance)


@pytest.mark.parametrize("shape", [(1, 3, 5000, 2, 1, 64), (1, 100, 130, 2, 2, 64), (1, 70, 90, 1, 1, 512)])
@pytest.mark.parametrize("dtype", TYPES[:2], ids=IDS[:2])
def test_scores_above_32_bits_are_no_rows_that_see_nothing(ctx, qrm, dtype, shape):
    n, lq, lk, heads, kv, d = shape
    q = torch.full((n, lq, heads, d), 2.0 ** 40, dtype=dtype, device="cuda")
    k, v = (torch.full((n, lk, kv, d), 2.0 ** 30, dtype=dtype, device="cuda") for _ in range(2))
    q[:, -1] = 0.0                                                             # (scores of zero: the mean of the values)
    o, lse = torch.empty_like(q), torch.empty((n, heads, lq), device="cuda")
    ctx.qrm_attention(desc_of(qrm, q, k, v, o, False, 2.0 ** 60), q, k, v, o, lse, None, None, 0)
    assert not bool(torch.isfinite(o[:, :-1]).any()) and not bool(torch.isneginf(lse[..., :-1]).any())
    assert float((o[:, -1].double() / 2.0 ** 30 - 1.0).abs().max()) <= lk * U + 2 * HALF[dtype]


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_values_that_are_not_finite_stay_in_their_image_and_key_head(ctx, qrm, dtype, bad):
    def both(dirty):
        c = Case(qrm, 2, 90, 100, 4, 2, 64, dtype, seed=9)
        if dirty:
            c.v[1, 99, 1, 5] = bad
            c.do[1, 3, 2, 7] = bad
        c.forward(ctx)
        c.backward(ctx)
        torch.cuda.synchronize()
        return c

    clean, dirty = both(False), both(True)
    for name in ("o", "dq", "dk", "dv"):
        a, b = getattr(clean, name).float(), getattr(dirty, name).float()
        own = (slice(1, 2), slice(None), slice(2, 4) if name in ("o", "dq") else slice(1, 2))
        assert not bool(torch.isfinite(b[own]).all()), name
        a[own], b[own] = 0, 0
        assert torch.equal(a, b), name


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", [(2, 100, 120, 4, 2, 64), (1, 40, 4000, 2, 1, 512), (1, 70, 90, 2, 2, 45)], ids=str)
def test_the_same_bits_from_call_to_call_and_beside_other_outputs(ctx, qrm, shape, dtype):
    c = Case(qrm, *shape, dtype, seed=2)
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    first = {k: getattr(c, k).clone() for k in ("o", "lse", "dq", "dk", "dv")}
    for wanted in (("dq", "dk", "dv"), ("dq",), ("dk",), ("dv",), ("dk", "dv")):
        for name in ("o", "dq", "dk", "dv"):
            getattr(c, name).fill_(7.0)
        c.forward(ctx, lse=wanted[0] == "dq")
        outs = [getattr(c, name) if name in wanted else None for name in ("dq", "dk", "dv")]
        ctx.qrm_attention_backward(c.desc, c.q, c.k, c.v, c.o, c.do, c.lse, *outs, *c.lens)
        torch.cuda.synchronize()
        for name in ("o", "lse") + wanted:
            assert torch.equal(first[name], getattr(c, name)), name
        for name in {"dq", "dk", "dv"} - set(wanted):
            assert bool((getattr(c, name) == 7.0).all()), name


def test_a_backward_pass_needs_no_forward_of_this_library(ctx, qrm):
    """o and lse may come from anywhere: the formulas say what they are."""
    c = Case(qrm, 2, 50, 60, 2, 2, 32, torch.float32, seed=12)
    o, lse, _ = at.attention(*c.args, c.scale)
    c.o.copy_(torch.from_numpy(o).float())
    c.lse.copy_(torch.from_numpy(lse).float())
    c.backward(ctx)
    torch.cuda.synchronize()
    c.check_backward()


def test_more_streams_than_workspaces(ctx, qrm):
    cases = [Case(qrm, 1, 2, 3000 + 100 * i, 2, 1, 64, torch.bfloat16, seed=i) for i in range(2 * qrm.QRM_MAX_STREAMS)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(2):
        for c, s in zip(cases, streams):
            ctx.qrm_attention(c.desc, c.q, c.k, c.v, c.o, c.lse, None, None, s)
            ctx.qrm_attention_backward(c.desc, c.q, c.k, c.v, c.o, c.do, c.lse, c.dq, c.dk, c.dv, None, None, s)
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        c.check_forward()
        c.check_backward()
        ctx.qrm_release_stream(s)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
@pytest.mark.parametrize("shape", [(3, 100, 700, 2, 1, 64), (3, 70, 300, 2, 2, 45), (2, 1, 5000, 8, 2, 128), (1, 260, 390, 1, 1, 512)])
def test_nothing_is_read_from_a_workspace_that_was_not_written(qrm, shape, dtype):
    """A workspace full of NaNs gives the bits of one of small numbers: splits that short images do not have, rows that are not there, copies of unaligned rows."""
    got = []
    for fill in (0x01, 0xFF):
        other = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
        other.qrm_diag_set_flags(qrm.binding.QRM_DIAG_POISON_WORKSPACE | fill << 8)
        n, lq, lk = shape[:3]
        c = Case(qrm, *shape, dtype, causal=True, q_len=[lq, max(1, lq // 3), 0][:n], k_len=[lk // 9, lk, lk // 2][:n], seed=8)
        c.forward(other)
        c.backward(other)
        torch.cuda.synchronize()
        got.append([t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv)])
        other.close()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert all(bool(torch.isfinite(t.float()).all()) for i, t in enumerate(got[0]) if i != 1)


def test_no_rows(ctx, qrm):
    c = Case(qrm, 2, 5, 0, 2, 1, 32, torch.bfloat16)
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    assert bool((c.o == 0).all()) and bool(torch.isneginf(c.lse).all()) and bool((c.dq == 0).all())
    c = Case(qrm, 2, 0, 5, 2, 1, 32, torch.bfloat16)
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    assert bool((c.dk == 0).all()) and bool((c.dv == 0).all())


def test_gradients_against_differences(ctx, qrm):
    """Of a loss sum(o * w): its change when an input moves, by central differences of the 64-bit oracle."""
    c = Case(qrm, 1, 9, 11, 4, 2, 8, torch.float32, causal=True, seed=4)
    c.forward(ctx)
    c.backward(ctx)
    torch.cuda.synchronize()
    w = f64(c.do)
    loss = lambda args: float((at.attention(*args, c.scale, True)[0] * w).sum())
    rng = np.random.default_rng(0)
    for index, name in enumerate(("dq", "dk", "dv")):
        got = f64(getattr(c, name))
        for _ in range(6):
            where = tuple(rng.integers(0, s) for s in c.args[index].shape)
            step, args = 1e-5, [t.copy() for t in c.args]
            args[index][where] += step
            up = loss(args)
            args[index][where] -= 2 * step
            slope = (up - loss(args)) / (2 * step)
            assert abs(slope - got[where]) <= 1e-5 * (1 + np.abs(got).max()) + 1e-8


def test_refusals(ctx, qrm):
    def refused(status, change=None, swap=None, **kw):
        args = dict(n=2, lq=5, lk=6, heads=4, kv=2, d=16, dtype=torch.bfloat16)
        c = Case(qrm, **{**args, **kw})
        for name, value in (change or {}).items():
            setattr(c.desc, name, value)
        ptr = lambda t: None if t is None else t.data_ptr()
        t = {k: ptr(getattr(c, k)) for k in ("q", "k", "v", "o", "do", "lse", "dq", "dk", "dv")}
        t.update(swap(t) if swap else {})
        import ctypes
        got = []
        if not swap or not {"do", "dq", "dk", "dv"} & set(swap(t)):
            got.append(ctx._lib.qrm_attention(ctx._h, ctypes.byref(c.desc), t["q"], t["k"], t["v"], None, None, t["o"], t["lse"], None))
        if not swap or "lse_forward" not in swap(t):
            got.append(ctx._lib.qrm_attention_backward(ctx._h, ctypes.byref(c.desc), t["q"], t["k"], t["v"], t["o"], t["do"], t["lse"], None, None, t["dq"], t["dk"], t["dv"], None))
        assert got and set(got) == {status}, got
        assert ctx.last_error()
        torch.cuda.synchronize()
        assert all(bool((getattr(c, k) == 7.0).all()) for k in ("dq", "dk", "dv")), "a refused call has written"

    bad = qrm.QRM_E_INVALID
    for change in (dict(N=-1), dict(Lq=-1), dict(Lk=-2), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(D=0), dict(type=3), dict(causal=2), dict(scale=0.0),
                   dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_row=15), dict(k_head=8), dict(o_image=64), dict(v_row=-32), dict(q_image=1 << 60)):
        refused(bad, change)
    for change in (dict(D=513), dict(Lk=(1 << 30) + 1), dict(Lq=1 << 29), dict(N=1 << 24)):
        refused(qrm.QRM_E_UNSUPPORTED, {**change, **{f"{t}_{s}": 0 for t in "qkvo" for s in ("row", "head", "image")}})
    refused(bad, swap=lambda t: dict(q=None))
    refused(bad, swap=lambda t: dict(k=None))
    refused(bad, swap=lambda t: dict(v=t["v"] + 1))
    refused(bad, swap=lambda t: dict(do=None))
    refused(bad, swap=lambda t: dict(dq=t["q"]))
    refused(bad, swap=lambda t: dict(dk=t["dv"]))
    refused(bad, swap=lambda t: dict(dq=None, dk=None, dv=None))
    assert ctx._lib.qrm_attention(ctx._h, None, None, None, None, None, None, None, None, None) == bad


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_single_rows_of_more_heads_than_a_launch_has_workgroups_for(ctx, qrm, dtype):
    """A workgroup of 512 threads takes the one row of a head and image: 2^23 of them for queries and as many for keys are 2^33 threads.  Said before anything is read."""
    import ctypes
    c = Case(qrm, 1, 1, 1, 1, 1, 512, dtype)
    c.desc.N = 1 << 23
    for t in "qkvo":
        for s in ("row", "head", "image"):
            setattr(c.desc, f"{t}_{s}", 0)
    p = {k: getattr(c, k).data_ptr() for k in ("q", "k", "v", "o", "do", "lse", "dq", "dk", "dv")}
    got = ctx._lib.qrm_attention_backward(ctx._h, ctypes.byref(c.desc), p["q"], p["k"], p["v"], p["o"], p["do"], p["lse"], None, None, p["dq"], p["dk"], p["dv"], None)
    assert got == qrm.QRM_E_UNSUPPORTED and "2^32" in ctx.last_error()


def test_the_binding_compares_tensors_with_their_descriptor(ctx, qrm):
    c = Case(qrm, 2, 5, 6, 4, 2, 16, torch.bfloat16)
    good = dict(d_q=c.q, d_k=c.k, d_v=c.v, d_o=c.o, d_lse=c.lse)
    ctx.qrm_attention(c.desc, **good)
    flat = lambda t: t.reshape(-1)
    ctx.qrm_attention(c.desc, flat(c.q), flat(c.k), flat(c.v), c.o, c.lse)
    wrong = [dict(d_q=c.q.float()), dict(d_k=c.k[:1]), dict(d_v=c.v.transpose(1, 2)), dict(d_o=c.o[:, :4]), dict(d_lse=c.lse[:1]), dict(d_lse=c.lse.bfloat16()), dict(d_q=c.q.cpu()),
             dict(d_q_len=torch.zeros(1, dtype=torch.int32, device="cuda")), dict(d_k_len=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(d_q=flat(c.q)[:-1])]
    for w in wrong:
        with pytest.raises(AssertionError):
            ctx.qrm_attention(c.desc, **{**good, **w})
    torch.cuda.synchronize()


@pytest.mark.parametrize("shape", [(2, 100, 120, 4, 2, 64), (1, 3, 5000, 4, 1, 128), (2, 70, 90, 1, 1, 45)], ids=str)
def test_streams_and_graphs(ctx, qrm, shape):
    """Eager on one stream, on another, and replays of a graph with other inputs between them."""
    c = Case(qrm, *shape, torch.bfloat16, causal=True, seed=8)
    names = ("o", "lse", "dq", "dk", "dv")

    def call(s):
        ctx.qrm_attention(c.desc, c.q, c.k, c.v, c.o, c.lse, *c.lens, s)
        ctx.qrm_attention_backward(c.desc, c.q, c.k, c.v, c.o, c.do, c.lse, c.dq, c.dk, c.dv, *c.lens, s)

    def eager():
        call(None)
        torch.cuda.synchronize()
        return {k: getattr(c, k).clone() for k in names}

    first, side = eager(), torch.cuda.Stream()
    call(side)
    side.synchronize()
    assert all(torch.equal(first[k], getattr(c, k)) for k in names)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(side)
    for k in range(3):
        c.q.mul_(0.75)
        c.do.mul_(1.5)
        want = eager()
        for name in names:
            getattr(c, name).fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[name], getattr(c, name)) for name in names)
