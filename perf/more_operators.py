"""Cases of the operators that an image decoder with attention needs beside those of perf/operators.py to be taught a key.

Three operators, each through the public entry points of paper_2509_02447_amd (include/qrm.h):

  attn       softmax attention of queries over keys and values, with what its backward pass needs   (qrm_attention)
  attn_grad  its backward pass, which computes the probabilities again                               (qrm_attention_backward)
  norm, clip the norm of all gradients of a network with the factor that clips it, and the gradients times that factor
             (qrm_adamw_grad_norm, qrm_adamw_scale_grads)

`own` false computes the plain forms: elementary torch operations in 32 bits, rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256           # a tensor of a network begins at a multiple of so many elements of the buffer
MAX_NORM = 1.0


# ---------------------------------------------------------------------------------------------- the cases
# lengths "none": all rows; "keys": of an image's keys only the first so many are there (padded prompts); "both": of its queries too.
# layout "rows": [images, rows, heads, dim]; "heads": [images, heads, rows, dim]; "packed": queries, keys and values of a row side by side.
def listed():
    attn, grad = dict(kind="attn"), dict(kind="attn_grad")
    return [
        # the attention of a decoder that makes four 256 x 256 images: 32 x 32 pixels, one head of all 512 channels
        dict(name="attn_4x1024_h1_d512_bf16", **attn, images=4, lq=1024, lk=1024, heads=1, kv=1, dim=512, type="bf16", causal=False,
             lengths="none", layout="rows"),
        # the same of 512 x 512 images
        dict(name="attn_4x4096_h1_d512_bf16", **attn, images=4, lq=4096, lk=4096, heads=1, kv=1, dim=512, type="bf16", causal=False,
             lengths="none", layout="rows"),
        # pixels that look at a padded prompt; one image has none
        dict(name="attn_8x4096_77_h8_d40_f16", **attn, images=8, lq=4096, lk=77, heads=8, kv=8, dim=40, type="f16", causal=False,
             lengths="keys", layout="rows"),
        # one new image token each for sixteen images under way, eight heads to a key's
        dict(name="attn_16x1_8191_h32_kv4_d128_bf16", **attn, images=16, lq=1, lk=8191, heads=32, kv=4, dim=128, type="bf16", causal=False,
             lengths="keys", layout="heads"),
        # odd maps in full precision, out of one projection's output
        dict(name="attn_3x2257_h6_d60_f32", **attn, images=3, lq=2257, lk=2257, heads=6, kv=6, dim=60, type="f32", causal=False,
             lengths="none", layout="packed"),
        # long rows of image tokens, each of which sees those before it
        dict(name="attn_2x8192_h16_kv4_d128_causal_bf16", **attn, images=2, lq=8192, lk=8192, heads=16, kv=4, dim=128, type="bf16",
             causal=True, lengths="none", layout="rows"),
        # a small decoder's attention in full precision, backward: latency
        dict(name="grad_4x256_h4_d16_f32", **grad, images=4, lq=256, lk=256, heads=4, kv=4, dim=16, type="f32", causal=False,
             lengths="none", layout="packed"),
        # the backward pass of the first case
        dict(name="grad_4x1024_h1_d512_bf16", **grad, images=4, lq=1024, lk=1024, heads=1, kv=1, dim=512, type="bf16", causal=False,
             lengths="none", layout="rows"),
        # ragged: padded queries and keys, odd rows, four heads to a key's, half precision
        dict(name="grad_5x777_1033_h8_kv2_d96_f16", **grad, images=5, lq=777, lk=1033, heads=8, kv=2, dim=96, type="f16", causal=True,
             lengths="both", layout="heads"),
        # long rows of image tokens, backward
        dict(name="grad_2x4096_h16_kv4_d128_causal_bf16", **grad, images=2, lq=4096, lk=4096, heads=16, kv=4, dim=128, type="bf16",
             causal=True, lengths="none", layout="rows"),
        # a small network's gradients in full precision: latency
        dict(name="norm_18_tensors_60k_f32", kind="norm", tensors=18, elements=60_000, grad="f32", unscale=False),
        # an image decoder's in 16 bits, added up over eight passes: the norm and the clipped gradients of their mean
        dict(name="clip_138_tensors_50m_bf16", kind="clip", tensors=138, elements=50_000_000, grad="bf16", unscale=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "attn_grad", "attn_grad", "attn_grad", "norm", "clip"])
    if kind in ("norm", "clip"):
        tensors = _log_int(rng, 1, 600)
        return dict(kind=kind, tensors=tensors, elements=max(tensors, _log_int(rng, 1_000, 50_000_000)), grad=rng.choice(["f32", "bf16", "f16"]),
                    unscale=rng.random() < 0.5)
    kv = rng.choice([1, 1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 1, 2, 4, 5, 8])
    dim = rng.choice([16, 32, 40, 64, 64, 80, 96, 128, 128, 160, 256, 512]) if rng.random() < 0.75 else rng.randint(3, 200)
    images = _log_int(rng, 1, 16)
    cells, lq = (2 * 16 * 8192 * 8192, 8192) if kind == "attn" else (2 * 16 * 4096 * 4096, 4096)
    lq, lk = _log_int(rng, 1, lq), _log_int(rng, 1, lq)
    if kind == "attn" and rng.random() < 0.3:                      # single tokens over long rows
        lq, lk = 1, _log_int(rng, 16, 32768)
    layout = rng.choice(["rows", "heads", "packed"])
    if layout == "packed":
        lk = lq
    most = min(cells, cells * 128 // dim) // (images * heads)
    while lq * lk > most:
        lq, lk = max(1, lq * 3 // 4), max(1, lk * 3 // 4)
    # (a row that sees one key alone has no gradient but rounding)
    if kind == "attn_grad":
        lq, lk = max(lq, 8), max(lk, 8)
        if layout == "packed":
            lq = lk = max(lq, lk)
    return dict(kind=kind, images=images, lq=lq, lk=lk, heads=heads, kv=kv, dim=dim, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                causal=rng.random() < 0.35, lengths=rng.choice(["none", "none", "keys", "both"]), layout=layout)


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case, rows, off):
    """Rows that are there: all of the first image's, none of the fourth's, between a quarter and all of the others'."""
    return [rows if i == 0 else 0 if i == 3 and off else max(1, math.ceil(rows * (0.25 + 0.75 * math.modf((i + off) * 0.6180339887498949)[0])))
            for i in range(case["images"])]


def _key_lengths(case):
    return None if case["lengths"] == "none" else _lengths(case, case["lk"], 1)


def _query_lengths(case):
    return _lengths(case, case["lq"], 0) if case["lengths"] == "both" else None


def _normal(shape, gen, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std)


def _place(case):
    """Queries, keys and values as views [images, rows, heads, dim] of buffers that lie as the case says."""
    n, lq, lk, h, kv, d = (case[k] for k in ("images", "lq", "lk", "heads", "kv", "dim"))
    new = lambda *shape: torch.empty(shape, dtype=TYPES[case["type"]], device="cuda")
    if case["layout"] == "packed":
        return new(n, lq, h + 2 * kv, d).split([h, kv, kv], dim=2)
    if case["layout"] == "heads":
        return tuple(new(n, heads, rows, d).transpose(1, 2) for heads, rows in ((h, lq), (kv, lk), (kv, lk)))
    return tuple(new(n, rows, heads, d) for heads, rows in ((h, lq), (kv, lk), (kv, lk)))


def _prepare_attn(case, gen):
    n, lq, lk, h, kv, d = (case[k] for k in ("images", "lq", "lk", "heads", "kv", "dim"))
    q, k, v = _place(case)
    # scores of a spread of one and a half; keys and values have a part that all rows share
    q.copy_(_normal(q.shape, gen, 1.4))
    k.copy_(_normal(k.shape, gen).add_(_normal((1, 1, kv, d), gen, 0.4)))
    v.copy_(_normal(v.shape, gen).add_(_normal((1, 1, kv, d), gen, 0.7)))
    st = dict(q=q, k=k, v=v)
    for name, lens in (("q_len", _query_lengths(case)), ("k_len", _key_lengths(case))):
        st[name] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["kind"] == "attn_grad":
        st["do"] = _normal((n, lq, h, d), gen, 0.02).to(q.dtype)
        kept = _plain_attn(dict(st, case=case))                    # what the forward pass has kept
        st.update(o=kept["o"], lse=kept["lse"])
    return st


def _tensor_sizes(case):
    """Sizes of a network's tensors: spread over five powers of e, odd ones among them, at least one element each."""
    t = case["tensors"]
    share = [math.exp(5.0 * math.modf(i * 0.6180339887498949)[0]) for i in range(t)]
    left = case["elements"] - t
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[-1] += case["elements"] - sum(sizes)
    return sizes


def _prepare_norm(case, gen):
    """The gradients lie in one buffer, zeros between them."""
    sizes, starts, at = _tensor_sizes(case), [], 0
    for s in sizes:
        starts.append(at)
        at += -(-s // BLOCK) * BLOCK
    grad = torch.zeros(at, dtype=torch.float32, device="cuda")
    # the norm is about three times what is allowed; the spread differs from tensor to tensor
    level = 3.0 / math.sqrt(case["elements"])
    for i, (s, a) in enumerate(zip(sizes, starts)):
        grad[a:a + s] = _normal((s,), gen, level * 2.0 ** (i % 4 - 2))
    st = dict(sizes=sizes, starts=starts, unscale=None)
    if case["unscale"]:                                            # gradients that were added up over eight passes
        grad.mul_(8.0)
        st["unscale"] = torch.full((1,), 1.0 / 8.0, device="cuda")
    st["grad"] = grad.to(TYPES[case["grad"]])
    return st


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_attn if case["kind"].startswith("attn") else _prepare_norm)(case, gen)


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
    case = st["case"]
    ctx = st["ctx"] = qrm.Context(rs=dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1))
    if case["kind"] in ("norm", "clip"):
        cut = lambda t: [t[a:a + s] for a, s in zip(st["starts"], st["sizes"])]
        st["grads"] = cut(st["grad"])
        st["out"] = dict(norm=torch.empty((1,), device="cuda"), scale=torch.empty((1,), device="cuda"))
        if case["kind"] == "clip":
            st["out"]["grad"] = torch.zeros_like(st["grad"])
            st["clipped"] = cut(st["out"]["grad"])
        flat = {k: torch.zeros(st["grad"].numel(), device="cuda") for k in ("param", "m", "v")}
        st["opt"] = qrm.AdamW(ctx, [dict(param=p, m=m, v=v) for p, m, v in zip(*(cut(flat[k]) for k in ("param", "m", "v")))],
                              grad_type=TYPES[case["grad"]])
        return
    n, lq, lk, h, kv, d = (case[k] for k in ("images", "lq", "lk", "heads", "kv", "dim"))
    strides = lambda t: (t.stride(1), t.stride(2), t.stride(0))    # of rows, heads, images
    typ = TYPES[case["type"]]
    o = st.get("o")
    if o is None:
        o = torch.empty((n, lq, h, d), dtype=typ, device="cuda")
    st["desc"] = qrm.attention_desc(N=n, Lq=lq, Lk=lk, heads=h, kv_heads=kv, D=d, dtype=typ, causal=case["causal"], scale=d ** -0.5,
                                    q=strides(st["q"]), k=strides(st["k"]), v=strides(st["v"]), o=strides(o))
    if case["kind"] == "attn":
        st["out"] = dict(o=o, lse=torch.empty((n, h, lq), dtype=torch.float32, device="cuda"))
    else:                                                          # gradients lie as what they are the gradients of
        st["out"] = dict(zip(("dq", "dk", "dv"), _place(case)))


# ---------------------------------------------------------------------------------------------- plain forms
def _hidden(case, q_len, k_len, device):
    """[images, 1, lq, lk]: whether a query does not see a key."""
    n, lq, lk = case["images"], case["lq"], case["lk"]
    i, j = torch.arange(lq, device=device).view(1, 1, lq, 1), torch.arange(lk, device=device).view(1, 1, 1, lk)
    ql = (torch.full((n,), lq, device=device) if q_len is None else q_len).view(n, 1, 1, 1)
    kl = (torch.full((n,), lk, device=device) if k_len is None else k_len).view(n, 1, 1, 1)
    hidden = (i >= ql) | (j >= kl)
    return hidden | (j > i + kl - ql) if case["causal"] else hidden


def _scores(st):
    """Scores [images, heads, lq, lk] in 32 bits, -inf where hidden, and the values [images, heads, lk, dim]."""
    case = st["case"]
    group = case["heads"] // case["kv"]
    by_head = lambda t, times: t.float().transpose(1, 2).repeat_interleave(times, dim=1)
    q, k, v = by_head(st["q"], 1), by_head(st["k"], group), by_head(st["v"], group)
    s = torch.matmul(q.contiguous(), k.transpose(2, 3).contiguous()) * case["dim"] ** -0.5
    if case["causal"] or case["lengths"] != "none":
        s = s.masked_fill_(_hidden(case, st["q_len"], st["k_len"], s.device), -math.inf)
    return s, q, k, v


def _plain_attn(st):
    s, _, _, v = _scores(st)
    top = s.amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)                  # (rows that see nothing)
    p = s.sub_(top).exp_()
    total = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p, v.contiguous()) / torch.where(total > 0, total, 1.0)
    return dict(o=o.transpose(1, 2).contiguous().to(st["q"].dtype), lse=(top + total.log()).squeeze(3))


def _plain_attn_grad(st):
    case = st["case"]
    n, lk, kv, d = (case[k] for k in ("images", "lk", "kv", "dim"))
    scale = d ** -0.5
    s, q, k, v = _scores(st)
    lse = st["lse"].unsqueeze(3)
    p = s.sub_(torch.where(lse == -math.inf, 0.0, lse)).exp_()     # (hidden: exp(-inf))
    do = st["do"].float().transpose(1, 2).contiguous()
    share = lambda t: t.view(n, kv, -1, lk, d).sum(dim=2)          # the heads that share a key's
    # (rows that see nothing pass no gradient on: their probabilities are zeros)
    dv = share(torch.matmul(p.transpose(2, 3).contiguous(), do))
    delta = (do * st["o"].float().transpose(1, 2)).sum(dim=3, keepdim=True)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_(delta).mul_(p).mul_(scale)
    dq = torch.matmul(ds, k.contiguous())
    dk = share(torch.matmul(ds.transpose(2, 3).contiguous(), q.contiguous()))
    return {name: t.transpose(1, 2).to(st["q"].dtype) for name, t in (("dq", dq), ("dk", dk), ("dv", dv))}


def _plain_norm(st):
    g = st["grad"]
    unscale = torch.ones((1,), device=g.device) if st["unscale"] is None else st["unscale"]
    norm = g.double().square().sum().sqrt().view(1) * unscale.double()   # a long sum
    scale = unscale.double() * torch.clamp_max(MAX_NORM / norm, 1.0)
    out = dict(norm=norm.float(), scale=scale.float())
    if st["case"]["kind"] == "clip":
        out["grad"] = (g.float() * out["scale"]).to(g.dtype)
    return out


# ---------------------------------------------------------------------------------------------- one pass
def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"attn": _plain_attn, "attn_grad": _plain_attn_grad, "norm": _plain_norm, "clip": _plain_norm}[kind](st)
    o, stream = st["out"], st["stream"]
    if kind == "attn":
        st["ctx"].qrm_attention(st["desc"], st["q"], st["k"], st["v"], o["o"], o["lse"], st["q_len"], st["k_len"], stream)
    elif kind == "attn_grad":
        st["ctx"].qrm_attention_backward(st["desc"], st["q"], st["k"], st["v"], st["o"], st["do"], st["lse"], o["dq"], o["dk"], o["dv"],
                                         st["q_len"], st["k_len"], stream)
    else:
        st["opt"].qrm_adamw_grad_norm(st["grads"], MAX_NORM, o["norm"], o["scale"], st["unscale"], stream)
        if kind == "clip":
            st["opt"].qrm_adamw_scale_grads(st["grads"], o["scale"], st["clipped"], stream)
    return o


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits, image by image and head by head."""
    st = _inputs(case, seed)
    return _exact_norm(st, case) if case["kind"] in ("norm", "clip") else _exact_attn(st, case)


def _exact_attn(st, case):
    n, lq, lk, h, kv, d = (case[k] for k in ("images", "lq", "lk", "heads", "kv", "dim"))
    grad, scale, group = case["kind"] == "attn_grad", 1.0 / math.sqrt(d), h // kv
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")
    if grad:
        out = dict(dq=zeros(n, lq, h, d), dk=zeros(n, lk, kv, d), dv=zeros(n, lk, kv, d))
    else:
        out = dict(o=zeros(n, lq, h, d), lse=zeros(n, h, lq) - math.inf)
    q_len, k_len = _query_lengths(case) or [lq] * n, _key_lengths(case) or [lk] * n
    for i in range(n):
        a, b = q_len[i], k_len[i]                                  # only rows that are there
        if a == 0 or b == 0:
            continue
        seen = torch.ones((a, b), dtype=torch.bool, device="cuda")
        if case["causal"]:
            seen = seen.tril(b - a)
        some = seen.any(dim=1)
        for j in range(h):
            q, k, v = st["q"][i, :a, j].double(), st["k"][i, :b, j // group].double(), st["v"][i, :b, j // group].double()
            e = torch.where(seen, (q @ k.t()) * scale, -math.inf)
            if not grad:
                lse = torch.logsumexp(e, dim=1)
                out["lse"][i, j, :a] = lse
                out["o"][i, :a, j] = torch.where(some[:, None], torch.exp(e - torch.where(some, lse, 0.0)[:, None]), 0.0) @ v
                continue
            p = torch.where(seen, torch.exp(e - torch.where(some, st["lse"][i, j, :a].double(), 0.0)[:, None]), 0.0)
            do = st["do"][i, :a, j].double()
            de = p * (do @ v.t() - (do * st["o"][i, :a, j].double()).sum(dim=1, keepdim=True))
            out["dv"][i, :b, j // group] += p.t() @ do
            out["dq"][i, :a, j] = scale * (de @ k)
            out["dk"][i, :b, j // group] += scale * (de.t() @ q)
    return out


def _exact_norm(st, case):
    factor = 1.0 if st["unscale"] is None else float(st["unscale"])
    parts = [st["grad"][a:a + s].double() for a, s in zip(st["starts"], st["sizes"])]
    norm = factor * math.sqrt(math.fsum(float(torch.dot(p, p)) for p in parts))
    scale = factor * (1.0 if norm <= MAX_NORM else MAX_NORM / norm)
    wide = lambda v: torch.tensor([v], dtype=torch.float64, device="cuda")
    out = dict(norm=wide(norm), scale=wide(scale))
    if case["kind"] == "clip":
        out["grad"] = st["grad"].double() * scale
    return out


# ---------------------------------------------------------------------------------------------- what a pass needs
def _pairs(case):
    """Pairs of a query and a key that it sees, over all images, and the rows that are there."""
    q_len, k_len = _query_lengths(case) or [case["lq"]] * case["images"], _key_lengths(case) or [case["lk"]] * case["images"]
    pairs = 0
    for a, b in zip(q_len, k_len):
        if not case["causal"]:
            pairs += a * b
        else:                                                      # query i sees max(0, i + 1 + b - a) keys
            seeing = min(a, b)
            pairs += seeing * (b - seeing + 1 + b) // 2
    return pairs, sum(q_len), sum(k_len)


def work(case):
    """Inputs read once, outputs written once; two products of matrices forward, five backward, over the pairs that see each other."""
    if case["kind"] in ("norm", "clip"):
        size = SIZE[case["grad"]]
        return dict(bytes=case["elements"] * size * (2 if case["kind"] == "clip" else 1) + 8, flops=case["elements"] * 2)
    pairs, queries, keys = _pairs(case)
    h, kv, d, size = case["heads"], case["kv"], case["dim"], SIZE[case["type"]]
    all_q, all_k = case["images"] * case["lq"], case["images"] * case["lk"]
    if case["kind"] == "attn":
        return dict(bytes=(queries * h + 2 * keys * kv + all_q * h) * d * size + all_q * h * 4, flops=pairs * h * d * 4)
    return dict(bytes=(3 * queries * h + 2 * keys * kv + all_q * h + 2 * all_k * kv) * d * size + queries * h * 4, flops=pairs * h * d * 10)
