"""Cases of the fine-tuning operators: what it takes to teach an image decoder to write the key that detection reads.

Three operators, each through the public entry points of paper_2509_02447_amd (include/qrm.h):

  norm       group norm with an activation over images of any size, channels last            (qrm_group_norm)
  norm_grad  its backward pass: gradients of the input, of the scale and of the bias         (qrm_group_norm_backward)
  adamw      one AdamW step over all tensors of a network, moments in 32 or in 8 bits        (qrm_adamw_step)
  loss       binary cross-entropy of the extractor's logits against a key, with the penalty for more wrong symbols than
             the Reed-Solomon code corrects, its gradient and the error counts               (qrm_message_loss)

`own` false computes the plain forms: elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
PRIM_POLY = {2: 0x7, 3: 0xB, 4: 0x13, 5: 0x25, 6: 0x43, 7: 0x89, 8: 0x11D}
BLOCK = 256           # elements of a tensor that share a scale where moments are held in 8 bits
NORM_EPS = 1e-6
BETA1, BETA2, ADAM_EPS, LR, STEP = 0.9, 0.999, 1e-8, 1e-4, 37


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # the innermost maps of a decoder that makes four 256 x 256 images: 32 x 32 pixels of 512 channels, latency counts
        dict(name="norm_4x1024_c512_bf16", kind="norm", images=4, pixels=32 * 32, channels=512, groups=32, type="bf16",
             act="silu", pitch=512),
        # ragged: 75 x 100 pixels, five channels a group, rows of a wider buffer (two maps side by side), full precision
        dict(name="norm_3x7500_c60_f32", kind="norm", images=3, pixels=75 * 100, channels=60, groups=12, type="f32",
             act="relu", pitch=92),
        # the outermost maps of the same decoder: four whole images at 128 channels
        dict(name="norm_4x65536_c128_bf16", kind="norm", images=4, pixels=256 * 256, channels=128, groups=32, type="bf16",
             act="silu", pitch=128),
        # the backward pass of a map half way
        dict(name="norm_grad_4x4096_c512_bf16", kind="norm_grad", images=4, pixels=64 * 64, channels=512, groups=32,
             type="bf16", act="silu", pitch=512),
        # an odd batch of odd maps, 37 x 61, without an activation, half precision
        dict(name="norm_grad_5x2257_c96_f16", kind="norm_grad", images=5, pixels=37 * 61, channels=96, groups=8, type="f16",
             act="none", pitch=96),
        # the backward pass of the outermost maps
        dict(name="norm_grad_4x65536_c128_bf16", kind="norm_grad", images=4, pixels=256 * 256, channels=128, groups=32,
             type="bf16", act="silu", pitch=128),
        # a small extractor's parameters in full precision: one launch's latency
        dict(name="adamw_18_tensors_60k_f32", kind="adamw", tensors=18, elements=60_000, param="f32", grad="f32",
             copy="none", bits=32, clip=False),
        # an image decoder: parameters kept in 32 bits, gradients in bf16, a bf16 copy for the next forward pass
        dict(name="adamw_138_tensors_50m_mixed", kind="adamw", tensors=138, elements=50_000_000, param="f32", grad="bf16",
             copy="bf16", bits=32, clip=True),
        # the same with moments in 8 bits
        dict(name="adamw_138_tensors_50m_8bit", kind="adamw", tensors=138, elements=50_000_000, param="f32", grad="bf16",
             copy="bf16", bits=8, clip=True),
        # a large network, everything in 32 bits
        dict(name="adamw_400_tensors_200m_f32", kind="adamw", tensors=400, elements=200_000_000, param="f32", grad="f32",
             copy="none", bits=32, clip=False),
        # the loss of a fine-tuning step: four images, one 48-bit key for all, RS(12,8) over GF(16)
        dict(name="loss_4_48bits", kind="loss", images=4, m=4, n=12, k=8, shared=True),
        # a large evaluation batch, a message for each image, 96 bits, RS(12,8) over GF(256)
        dict(name="loss_16384_96bits", kind="loss", images=16384, m=8, n=12, k=8, shared=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "adamw", "adamw", "loss"])
    if kind in ("norm", "norm_grad"):
        groups = rng.choice([1, 2, 4, 8, 12, 16, 32, 32])
        each = _log_int(rng, 1, 32)                             # channels of a group
        channels = min(groups * each, 1024 // groups * groups)
        most = 4 * 65536 * 128                                   # elements of the largest listed case
        images = _log_int(rng, 1, 16)
        pixels = _log_int(rng, 1, min(65536, max(1, most // (channels * images))))
        pitch = channels + (rng.choice([8, 32, channels]) if rng.random() < 0.25 else 0)
        typ = rng.choice(["bf16", "bf16", "f16", "f32"])
        if typ == "f32":
            pixels = max(1, pixels // 2)
        if kind == "norm_grad":                                  # a group of one or two values has no gradient but rounding
            pixels = max(pixels, -(-8 * groups // channels))
        return dict(kind=kind, images=images, pixels=pixels, channels=channels, groups=groups, type=typ,
                    act=rng.choice(["silu", "silu", "relu", "none"]), pitch=pitch)
    if kind == "adamw":
        param, grad, copy = rng.choice([("f32", "f32", "none"), ("f32", "bf16", "bf16"), ("f32", "f16", "f16"),
                                        ("bf16", "bf16", "none"), ("f32", "f32", "bf16")])
        tensors = _log_int(rng, 1, 400)
        return dict(kind="adamw", tensors=tensors, elements=max(tensors, _log_int(rng, 1_000, 100_000_000)), param=param,
                    grad=grad, copy=copy, bits=rng.choice([32, 8]), clip=rng.random() < 0.5)
    m = rng.choice([2, 3, 4, 4, 5, 6, 8, 8])
    n = rng.randint(3, min((1 << m) - 1, 128 // m))
    return dict(kind="loss", images=_log_int(rng, 1, 16384), m=m, n=n, k=n - 2 * rng.randint(1, (n - 1) // 2),
                shared=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs
def _tensor_sizes(case):
    """Sizes of a network's tensors: spread over five powers of e, odd ones among them, at least one element each."""
    t = case["tensors"]
    share = [math.exp(5.0 * math.modf(i * 0.6180339887498949)[0]) for i in range(t)]
    left = case["elements"] - t
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[-1] += case["elements"] - sum(sizes)
    return sizes


def _normal(shape, gen, std=1.0, mean=0.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).add_(mean)


def _prepare_norm(case, gen):
    n, p, c, pitch = case["images"], case["pixels"], case["channels"], case["pitch"]
    typ = TYPES[case["type"]]
    level, spread = _normal((1, 1, c), gen, 1.5), torch.rand((1, 1, c), generator=gen, device="cuda").mul_(2.7).add_(0.3)
    # the map is the first `channels` of a buffer that may be wider; its results are a map of their own
    wide = torch.zeros((n, p, pitch), dtype=typ, device="cuda")
    wide[:, :, :c] = _normal((n, p, c), gen).mul_(spread).add_(level)
    st = dict(x=wide[:, :, :c], gamma=_normal((c,), gen, 0.2, 1.0), beta=_normal((c,), gen, 0.2))
    if case["kind"] == "norm_grad":
        st["dy"] = _normal((n, p, c), gen, 0.05).to(typ)
        xg = st["x"].float().view(n, p, case["groups"], -1)      # what the forward pass has kept
        st["mean"] = xg.mean(dim=(1, 3))
        var = (xg - st["mean"].view(n, 1, -1, 1)).square().mean(dim=(1, 3))
        st["rstd"] = (var + NORM_EPS).rsqrt()
    return st


def _prepare_adamw(case, gen):
    """The tensors of a network lie in one buffer of each kind, every one from a multiple of BLOCK elements on."""
    sizes = _tensor_sizes(case)
    starts, at = [], 0
    for s in sizes:
        starts.append(at)
        at += -(-s // BLOCK) * BLOCK
    total = at
    live = torch.zeros(total, dtype=torch.float32, device="cuda")
    # the spread of a tensor's gradients differs from tensor to tensor, that of its elements too
    strength = torch.zeros(total, dtype=torch.float32, device="cuda")
    decay = torch.zeros((total // BLOCK, 1), dtype=torch.float32, device="cuda")
    for i, (s, a) in enumerate(zip(sizes, starts)):
        live[a:a + s] = 1.0
        strength[a:a + s] = 10.0 ** -(2.0 + i % 4)
        if s > 256:                                              # weight decay on matrices and filters only
            decay[a // BLOCK:-(-(a + s) // BLOCK)] = 0.01
    strength.mul_(live)
    st = dict(sizes=sizes, starts=starts, decay=decay)
    st["param"] = _normal((total,), gen, 0.05).mul_(live).to(TYPES[case["param"]])
    st["grad"] = _normal((total,), gen).mul_(strength).to(TYPES[case["grad"]])
    m = _normal((total,), gen, 0.3).mul_(strength)
    u = torch.rand((total,), generator=gen, device="cuda").mul_(0.3).add_(0.02).mul_(strength)
    if case["bits"] == 32:
        st["m"], st["v"] = m, u.square_()
    else:
        st["m"], st["m_scale"] = _pack_m(m.view(-1, BLOCK))
        st["v"], st["v_scale"] = _pack_u(u.view(-1, BLOCK))
    st["copy"] = None if case["copy"] == "none" else torch.zeros(total, dtype=TYPES[case["copy"]], device="cuda")
    st["scale"] = torch.full((1,), 0.75, device="cuda") if case["clip"] else None
    return st


def _prepare_loss(case, gen):
    n, bits = case["images"], case["m"] * case["n"]
    target = torch.randint(0, 2, (1 if case["shared"] else n, bits), generator=gen, device="cuda", dtype=torch.uint8)
    # logits of a half-taught network: most on the right side, some far off
    logits = _normal((n, bits), gen, 2.0).add_((target.float() * 2 - 1) * 2.5)
    return dict(logits=logits, target=target)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = {"norm": _prepare_norm, "norm_grad": _prepare_norm, "adamw": _prepare_adamw, "loss": _prepare_loss}
    return make[case["kind"]](case, gen)


def prepare(case, seed):
    st = _inputs(case, seed)
    st.update(case=case, stream=torch.cuda.current_stream())
    if own:
        _handles(st)
    torch.cuda.synchronize()
    return st


def _handles(st):
    """The context, the plan and the result buffers that a program keeps from step to step."""
    import paper_2509_02447_amd as qrm
    case, kind = st["case"], st["case"]["kind"]
    if kind == "loss":
        m, n, bits = case["m"], case["images"], case["m"] * case["n"]
        ctx = st["ctx"] = qrm.Context(rs=dict(m=m, prim_poly=PRIM_POLY[m], n=case["n"], k=case["k"], fcr=1))
        st["out"] = dict(loss=torch.empty((1,), device="cuda"), grad=torch.empty((n, bits), device="cuda"),
                         bit_errors=torch.empty((n,), dtype=torch.int32, device="cuda"),
                         symbol_errors=torch.empty((n,), dtype=torch.int32, device="cuda"))
        return
    ctx = st["ctx"] = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    if kind == "adamw":
        cut = lambda t: [None] * case["tensors"] if t is None else [t[a:a + s] for a, s in zip(st["starts"], st["sizes"])]
        scales = lambda t: [t[a // BLOCK:-(-(a + s) // BLOCK)] for a, s in zip(st["starts"], st["sizes"])]
        eight = case["bits"] == 8
        rows = zip(cut(st["param"]), cut(st["m"].view(-1)), cut(st["v"].view(-1)), cut(st["copy"]),
                   scales(st["m_scale"]) if eight else cut(None), scales(st["v_scale"]) if eight else cut(None), st["sizes"])
        st["opt"] = qrm.AdamW(ctx, [dict(param=p, m=m, v=v, copy=c, m_scale=ms, v_scale=vs, weight_decay=0.01 if s > 256 else 0.0)
                                    for p, m, v, c, ms, vs, s in rows], grad_type=TYPES[case["grad"]])
        st["grads"] = cut(st["grad"])
        if eight:
            st["out"] = {k: torch.empty_like(st["param"], dtype=torch.bfloat16) for k in ("m", "v")}
        return
    n, p, c, g = case["images"], case["pixels"], case["channels"], case["groups"]
    st["desc"] = qrm.group_norm_desc(N=n, P=p, C=c, groups=g, dtype=TYPES[case["type"]], act=case["act"], eps=NORM_EPS,
                                     x_pixel=case["pitch"], x_image=p * case["pitch"])
    keep = dict(dtype=torch.float32, device="cuda")
    if kind == "norm":
        st["out"] = dict(y=torch.empty((n, p, c), dtype=TYPES[case["type"]], device="cuda"),
                         mean=torch.empty((n, g), **keep), rstd=torch.empty((n, g), **keep))
    else:                                                        # the input's gradient lies as the input does
        wide = torch.empty((n, p, case["pitch"]), dtype=TYPES[case["type"]], device="cuda")
        st["out"] = dict(dx=wide[:, :, :c], dgamma=torch.empty((c,), **keep), dbeta=torch.empty((c,), **keep))


# ---------------------------------------------------------------------------------------------- plain forms
def _act(z, act):
    return z * torch.sigmoid(z) if act == "silu" else torch.clamp_min(z, 0.0) if act == "relu" else z


def _plain_norm(st):
    case, x = st["case"], st["x"]
    n, p, c, g = case["images"], case["pixels"], case["channels"], case["groups"]
    xg = x.float().view(n, p, g, c // g)
    mean = xg.mean(dim=(1, 3))
    d = xg - mean.view(n, 1, g, 1)
    rstd = torch.rsqrt(d.square().mean(dim=(1, 3)) + NORM_EPS)
    z = (d * rstd.view(n, 1, g, 1)).view(n, p, c) * st["gamma"] + st["beta"]
    return dict(y=_act(z, case["act"]).to(x.dtype), mean=mean, rstd=rstd)


def _plain_norm_grad(st):
    case, x = st["case"], st["x"]
    n, p, c, g = case["images"], case["pixels"], case["channels"], case["groups"]
    mean, rstd = st["mean"].view(n, 1, g, 1), st["rstd"].view(n, 1, g, 1)
    xhat = ((x.float().view(n, p, g, c // g) - mean) * rstd).view(n, p, c)
    dz = st["dy"].float()
    if case["act"] != "none":
        z = xhat * st["gamma"] + st["beta"]
        if case["act"] == "silu":
            s = torch.sigmoid(z)
            dz = dz * (s * (1.0 + z * (1.0 - s)))
        else:
            dz = dz * (z > 0)
    dgamma, dbeta = (dz * xhat).sum(dim=(0, 1)), dz.sum(dim=(0, 1))
    dh, hg = (dz * st["gamma"]).view(n, p, g, c // g), xhat.view(n, p, g, c // g)
    a, b = dh.mean(dim=(1, 3), keepdim=True), (dh * hg).mean(dim=(1, 3), keepdim=True)
    dx = (dh - a - hg * b) * rstd
    return dict(dx=dx.view(n, p, c).to(x.dtype), dgamma=dgamma, dbeta=dbeta)


def _pack_m(m):
    """[blocks,256] -> int8 codes c with m = scale * c |c| / 127^2, scale the largest |m| of a block."""
    scale = m.abs().amax(dim=1, keepdim=True)
    part = torch.where(scale > 0, m.abs() / scale, 0.0)
    code = torch.round(torch.sqrt(part) * 127.0) * torch.sign(m)
    return code.to(torch.int8), scale.view(-1)


def _pack_u(u):
    """[blocks,256] of roots u = sqrt(v) -> uint8 codes c with u = scale * c^2 / 255^2; a root above zero keeps a code above zero."""
    scale = u.amax(dim=1, keepdim=True)
    part = torch.where(scale > 0, u / scale, 0.0)
    code = torch.maximum(torch.round(torch.sqrt(part) * 255.0), (u > 0).to(u.dtype))
    return code.to(torch.uint8), scale.view(-1)


def _unpack_m(code, scale):
    c = code.to(scale.dtype)
    return scale.view(-1, 1) * (c * c.abs() * (1.0 / 16129.0))


def _unpack_u(code, scale):
    c = code.to(scale.dtype)
    return scale.view(-1, 1) * (c * c * (1.0 / 65025.0))


def _plain_adamw(st):
    case = st["case"]
    p, g = st["param"].float().view(-1, BLOCK), st["grad"].float().view(-1, BLOCK)
    if st["scale"] is not None:
        g = g * st["scale"]
    eight = case["bits"] == 8
    m = _unpack_m(st["m"], st["m_scale"]) if eight else st["m"].view(-1, BLOCK)
    v = _unpack_u(st["v"], st["v_scale"]).square() if eight else st["v"].view(-1, BLOCK)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    root = torch.sqrt(v)
    p = p * (1.0 - LR * st["decay"]) - (LR / (1.0 - BETA1 ** STEP)) * m / (root * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + ADAM_EPS)
    st["param"].copy_(p.view(-1))
    out = dict(param=st["param"])
    if eight:
        st["m"], st["m_scale"] = _pack_m(m)
        st["v"], st["v_scale"] = _pack_u(root)
        # 8-bit moments are returned as the values they stand for, in 16 bits: a step of their codes is coarser than those
        out["m"] = _unpack_m(st["m"], st["m_scale"]).view(-1).to(torch.bfloat16)
        out["v"] = _unpack_u(st["v"], st["v_scale"]).square().view(-1).to(torch.bfloat16)
    else:
        st["m"].copy_(m.view(-1))
        st["v"].copy_(v.view(-1))
        out.update(m=st["m"], v=st["v"])
    if st["copy"] is not None:
        st["copy"].copy_(p.view(-1))
        out["copy"] = st["copy"]
    return out


RS_WEIGHT = 1.0


def _plain_loss(st):
    case, z = st["case"], st["logits"]
    n, m, symbols, t = case["images"], case["m"], case["n"], (case["n"] - case["k"]) // 2
    sign = st["target"].float() * 2.0 - 1.0                      # +1 / -1: the side a bit has to be on
    x = z * sign
    e = torch.exp(-x.abs())
    bce = torch.clamp_min(-x, 0.0) + torch.log1p(e)              # -log sigmoid(x)
    miss = torch.where(x >= 0, e, torch.ones_like(e)) / (1.0 + e)   # sigmoid(-x): the chance that the bit is wrong
    right = torch.exp(-bce.view(n, symbols, m).sum(dim=2))       # the chance that all bits of a symbol are right
    over = torch.clamp_min((1.0 - right).sum(dim=1) - t, 0.0)    # expected wrong symbols beyond what the code corrects
    loss = bce.sum() / (n * symbols * m) + RS_WEIGHT * over.square().sum() / n
    pull = 1.0 / (n * symbols * m) + (2.0 * RS_WEIGHT / n) * over.view(n, 1, 1) * right.view(n, symbols, 1)
    grad = -sign * miss * pull.expand(n, symbols, m).reshape(n, symbols * m)
    wrong = (z > 0) != (sign > 0)
    return dict(loss=loss.view(1), grad=grad, bit_errors=wrong.sum(dim=1, dtype=torch.int32),
                symbol_errors=wrong.view(n, symbols, m).any(dim=2).sum(dim=1, dtype=torch.int32))


# ---------------------------------------------------------------------------------------------- one pass
def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if not own:
        return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "adamw": _plain_adamw, "loss": _plain_loss}[kind](st)
    ctx, stream = st["ctx"], st["stream"]
    if kind == "norm":
        o = st["out"]
        ctx.qrm_group_norm(st["desc"], st["x"], st["gamma"], st["beta"], o["y"], o["mean"], o["rstd"], stream)
        return o
    if kind == "norm_grad":
        o = st["out"]
        ctx.qrm_group_norm_backward(st["desc"], st["x"], st["dy"], st["gamma"], st["beta"], st["mean"], st["rstd"],
                                    o["dx"], o["dgamma"], o["dbeta"], stream)
        return o
    if kind == "adamw":
        st["opt"].qrm_adamw_step(st["grads"], STEP, LR, BETA1, BETA2, ADAM_EPS, st["scale"], stream)
        out = dict(param=st["param"], m=st["m"], v=st["v"])
        if case["bits"] == 8:                                    # the values that the codes stand for
            ctx.qrm_unpack_moment(0, st["m"], st["m_scale"], st["m"].numel(), st["out"]["m"], stream)
            ctx.qrm_unpack_moment(1, st["v"], st["v_scale"], st["v"].numel(), st["out"]["v"], stream)
            out.update(st["out"])
        if st["copy"] is not None:
            out["copy"] = st["copy"]
        return out
    o = st["out"]
    ctx.qrm_message_loss(st["logits"], st["target"], st["target"].shape[0], case["images"], case["m"] * case["n"], RS_WEIGHT,
                         o["loss"], o["grad"], o["bit_errors"], o["symbol_errors"], stream)
    return o


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits; gradients by differentiating the forward definition instead of the formulas above."""
    st = _inputs(case, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm, "adamw": _exact_adamw, "loss": _exact_loss}[case["kind"]](st, case)


def _exact_norm(st, case):
    grad = case["kind"] == "norm_grad"
    n, p, g = case["images"], case["pixels"], case["groups"]
    x = st["x"].double().contiguous().requires_grad_(grad)
    gamma, beta = st["gamma"].double().requires_grad_(grad), st["beta"].double().requires_grad_(grad)
    with torch.set_grad_enabled(grad):
        # group by group: mean and variance (the biased one) over the group's channels and all pixels, from the input again
        rows = x.reshape(n, p, g, -1).transpose(1, 2).reshape(n, g, -1)
        mean = rows.sum(dim=2) / rows.shape[2]
        var = (rows - mean[:, :, None]).pow(2).sum(dim=2) / rows.shape[2]
        unit = (rows - mean[:, :, None]) / (var + NORM_EPS).sqrt()[:, :, None]
        z = unit.reshape(n, g, p, -1).transpose(1, 2).reshape(n, p, -1) * gamma + beta
        y = z / (1.0 + torch.exp(-z)) if case["act"] == "silu" else torch.where(z > 0, z, 0.0 * z) if case["act"] == "relu" else z
        if not grad:
            return dict(y=y, mean=mean, rstd=1.0 / (var + NORM_EPS).sqrt())
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), st["dy"].double())
    return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)


def _exact_adamw(st, case):
    wide = lambda t: t.double().view(-1, BLOCK)
    p, g = wide(st["param"]), wide(st["grad"])
    if st["scale"] is not None:
        g = g * st["scale"].double()
    if case["bits"] == 8:
        code = st["m"].double()
        m = st["m_scale"].double()[:, None] * code.sign() * (code / 127.0) ** 2
        v = (st["v_scale"].double()[:, None] * (st["v"].double() / 255.0) ** 2) ** 2
    else:
        m, v = wide(st["m"]), wide(st["v"])
    m = m + (1.0 - BETA1) * (g - m)
    v = v + (1.0 - BETA2) * (g ** 2 - v)
    step = (m / (1.0 - BETA1 ** STEP)) / ((v / (1.0 - BETA2 ** STEP)).sqrt() + ADAM_EPS)
    p = p - LR * st["decay"].double() * p - LR * step
    if case["bits"] == 8:
        top = m.abs().amax(dim=1, keepdim=True)
        code = torch.floor((m.abs() / top.clamp_min(1e-300)).sqrt() * 127.0 + 0.5)
        m = m.sign() * top * code ** 2 / 127.0 ** 2
        u = v.sqrt()
        top = u.amax(dim=1, keepdim=True)
        code = torch.floor((u / top.clamp_min(1e-300)).sqrt() * 255.0 + 0.5).clamp_min(1.0)
        v = torch.where(u > 0, (top * code ** 2 / 255.0 ** 2) ** 2, 0.0)
    out = dict(param=p.view(-1), m=m.view(-1), v=v.view(-1))
    if st["copy"] is not None:
        out["copy"] = p.view(-1)
    return out


def _exact_loss(st, case):
    n, t = case["images"], (case["n"] - case["k"]) // 2
    z = st["logits"].double().requires_grad_(True)
    want = st["target"].double().expand(n, -1)
    chance = torch.where(want > 0.5, torch.sigmoid(z), torch.sigmoid(-z))     # of the right bit
    bce = torch.where(want > 0.5, torch.nn.functional.softplus(-z, threshold=700.0), torch.nn.functional.softplus(z, threshold=700.0))
    wrong = (1.0 - chance.view(n, case["n"], case["m"]).prod(dim=2)).sum(dim=1)
    loss = bce.mean() + RS_WEIGHT * torch.relu(wrong - t).pow(2).mean()
    grad, = torch.autograd.grad(loss, z)
    return dict(loss=loss.detach().view(1), grad=grad, bit_errors=None, symbol_errors=None)


# ---------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Inputs read once, outputs written once; operations of the formulas, an exponential or a root counted as one."""
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        cells = case["images"] * case["pixels"] * case["channels"]
        kept = case["images"] * case["groups"] * 8 + case["channels"] * 8
        if kind == "norm":
            return dict(bytes=cells * 2 * SIZE[case["type"]] + kept, flops=cells * 12)
        return dict(bytes=cells * 3 * SIZE[case["type"]] + kept + case["channels"] * 8, flops=cells * 25)
    if kind == "adamw":
        each = 2 * SIZE[case["param"]] + SIZE[case["grad"]] + SIZE.get(case["copy"], 0)
        # 8-bit moments: codes and scales read and written, and their values written in 16 bits
        each += 16 if case["bits"] == 32 else 4 + 16.0 / BLOCK + 4
        return dict(bytes=case["elements"] * each, flops=case["elements"] * (16 if case["bits"] == 32 else 32))
    cells = case["images"] * case["m"] * case["n"]
    target = cells // case["images"] if case["shared"] else cells
    return dict(bytes=cells * 8 + target + case["images"] * 8 + 4, flops=cells * 15)
