"""Teaches a small image decoder to write a key that the detector reads (Section 4.2: the decoder is fine-tuned, the extractor stays as it is).

The steps are those of the paper in small: images of a decoder made of group-norm blocks, the frozen extractor's logits, the message loss against a
Reed-Solomon code word, a term that keeps the images near what they were, AdamW with a warm-up.  Then the images go through the detector as
any others do: crop, extractor, Reed-Solomon decoding and the comparison with the key.

The group norms, the message loss and the optimiser are the library's (qrm_group_norm, qrm_group_norm_backward, qrm_message_loss, qrm_adamw_step); convolutions are
plain matrix products of torch, which also differentiates them.  With --attention the decoder's pixels also look at each other between the residual blocks
(qrm_attention, qrm_attention_backward); with --clip the gradients' norm is bounded (qrm_adamw_grad_norm).

    python examples/finetune_decoder.py [--steps 200] [--bits 8] [--attention] [--clip 1.0]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2509_02447_amd as qrm  # noqa: E402

CODE = dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1)
BITS = CODE["m"] * CODE["n"]
SIDE, CHANNELS, BLOCKS = 32, 32, 4          # of the images, the extractor's channels and blocks
WHITEN = 1e-5                               # of the strongest axis: the least that an axis counts for
MEAN, STD = (0.485, 0.456, 0.406), (0.229, 0.224, 0.225)


class Once(torch.autograd.Function):
    """A gradient as it is.  The library has first derivatives alone: who differentiates one again, with respect to what it was computed of,
    is told so instead of losing its share."""

    @staticmethod
    def forward(fn, grad, *of):
        return grad.view_as(grad)

    @staticmethod
    def backward(fn, *_):
        raise RuntimeError("the library's gradients cannot be differentiated again")


class NormAct(torch.autograd.Function):
    """SiLU of a group norm over x [N,H,W,C], channels last, through the library."""

    @staticmethod
    def forward(fn, x, gamma, beta, ctx, groups):
        n, h, w, c = x.shape
        x = x.contiguous()
        fn.desc = qrm.group_norm_desc(n, h * w, c, groups, x.dtype, "silu")
        y, mean, rstd = torch.empty_like(x), x.new_empty((n, groups), dtype=torch.float32), x.new_empty((n, groups), dtype=torch.float32)
        ctx.qrm_group_norm(fn.desc, x, gamma, beta, y, mean, rstd)
        fn.ctx = ctx
        fn.save_for_backward(x, gamma, beta, mean, rstd)
        return y

    @staticmethod
    def backward(fn, dy):
        x, gamma, beta, mean, rstd = fn.saved_tensors
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
        fn.ctx.qrm_group_norm_backward(fn.desc, x, dy.contiguous(), gamma, beta, mean, rstd, dx, dgamma, dbeta)
        return *(Once.apply(g, x, gamma, beta, dy) for g in (dx, dgamma, dbeta)), None, None


class Attend(torch.autograd.Function):
    """Softmax attention of q [N,Lq,H,D] over k, v [N,Lk,KV,D] through the library; lengths i32 [N] of queries and keys, or None."""

    @staticmethod
    def forward(fn, q, k, v, ctx, causal, q_len, k_len):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        n, lq, heads, d = q.shape
        fn.desc = qrm.attention_desc(n, lq, k.shape[1], heads, k.shape[2], d, q.dtype, causal)
        o, lse = torch.empty_like(q), q.new_empty((n, heads, lq), dtype=torch.float32)
        ctx.qrm_attention(fn.desc, q, k, v, o, lse, q_len, k_len)
        fn.ctx, fn.lens = ctx, (q_len, k_len)
        fn.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(fn, do):
        q, k, v, o, lse = fn.saved_tensors
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        fn.ctx.qrm_attention_backward(fn.desc, q, k, v, o, do.contiguous(), lse, dq, dk, dv, *fn.lens)
        return *(Once.apply(g, q, k, v, do) for g in (dq, dk, dv)), None, None, None, None


class MessageLoss(torch.autograd.Function):
    """The library's message loss of logits [N,BITS] against one target for all; its gradient comes with it."""

    @staticmethod
    def forward(fn, logits, target, ctx, rs_weight, errors):
        loss, grad = logits.new_empty(1), torch.empty_like(logits)
        ctx.qrm_message_loss(logits.contiguous(), target, 1, logits.shape[0], BITS, rs_weight, loss, grad, errors)
        fn.save_for_backward(logits, grad)
        return loss[0]

    @staticmethod
    def backward(fn, g):
        logits, grad = fn.saved_tensors
        return Once.apply(g * grad, logits, g), None, None, None, None


def conv3x3(x, w):
    """3 x 3 convolution of x [N,H,W,C] with w [9 C, C_out], zero padding: one matrix product."""
    n, h, wd, c = x.shape
    p = torch.nn.functional.pad(x, (0, 0, 1, 1, 1, 1))
    taps = torch.cat([p[:, i:i + h, j:j + wd] for i in range(3) for j in range(3)], dim=3)
    return (taps.reshape(n * h * wd, 9 * c) @ w).view(n, h, wd, -1)


class Decoder:
    """Latents [N,16,16,8] -> images [N,32,32,3] in 0..1: two residual blocks, doubling, one more block; with attention between the two of four heads of 16."""

    def __init__(self, gen, attention=False):
        def conv(cin, cout, gain=1.0):
            return (torch.randn((9 * cin, cout), generator=gen, device="cuda") * (gain * math.sqrt(2.0 / (9 * cin)))).requires_grad_()

        ones, zeros = (lambda c: torch.ones(c, device="cuda").requires_grad_()), (lambda c: torch.zeros(c, device="cuda").requires_grad_())
        self.first = conv(8, 64)
        self.blocks = [(ones(64), zeros(64), conv(64, 64, 0.5)) for _ in range(2)]
        self.up = (ones(64), zeros(64), conv(64, 32))
        self.last = (ones(32), zeros(32), conv(32, 3, 0.5))
        self.params = [self.first] + [p for b in self.blocks for p in b] + list(self.up) + list(self.last)
        self.look = None
        if attention:
            mix = lambda cout, gain: (torch.randn((64, cout), generator=gen, device="cuda") * (gain / 8.0)).requires_grad_()
            self.look = (ones(64), zeros(64), mix(192, 1.0), mix(64, 0.5))
            self.params += list(self.look)

    def __call__(self, z, ctx):
        x = conv3x3(z, self.first)
        for i, (gamma, beta, w) in enumerate(self.blocks):
            x = x + conv3x3(NormAct.apply(x, gamma, beta, ctx, 16), w)
            if self.look is not None and i == 0:
                gamma, beta, into, out = self.look
                n, h, wd, _ = x.shape
                q, k, v = (NormAct.apply(x, gamma, beta, ctx, 16).reshape(n, h * wd, 64) @ into).view(n, h * wd, 3, 4, 16).unbind(2)
                x = x + (Attend.apply(q, k, v, ctx, False, None, None).reshape(n, h * wd, 64) @ out).view(n, h, wd, 64)
        x = NormAct.apply(x, self.up[0], self.up[1], ctx, 16)
        x = conv3x3(x.repeat_interleave(2, dim=1).repeat_interleave(2, dim=2), self.up[2])
        return torch.sigmoid(conv3x3(NormAct.apply(x, self.last[0], self.last[1], ctx, 8), self.last[2]))


def extractor_weights(rng):
    """A random extractor in the layout of qrm_create: conv blocks with scale and bias, a final convolution, a linear layer."""
    conv = [rng.normal(0.0, math.sqrt(2.0 / 27), (CHANNELS, 3, 3, 3))]
    conv += [rng.normal(0.0, math.sqrt(2.0 / (9 * CHANNELS)), (CHANNELS, CHANNELS, 3, 3)) for _ in range(BLOCKS - 1)]
    conv.append(rng.normal(0.0, math.sqrt(2.0 / (9 * CHANNELS)), (BITS, CHANNELS, 3, 3)))
    w = dict(in_ch=3, n_blocks=BLOCKS, channels=CHANNELS, n_bits=BITS, scale=np.ones(BLOCKS * CHANNELS), bias=np.zeros(BLOCKS * CHANNELS),
             lin_w=rng.normal(0.0, math.sqrt(2.0 / BITS), (BITS, BITS)), lin_b=np.zeros(BITS), mean=np.array(MEAN), std=np.array(STD))
    w["conv_w"] = np.concatenate([c.reshape(-1) for c in conv])
    return {k: v.astype(np.float32) if isinstance(v, np.ndarray) else v for k, v in w.items()}


class Extractor:
    """The same network for images [N,H,W,3] in 0..1, differentiable in its input."""

    def __init__(self, w):
        self.mean, self.std = (torch.tensor(v, device="cuda") for v in (MEAN, STD))
        at, self.convs = 0, []
        for cout, cin in [(CHANNELS, 3)] + [(CHANNELS, CHANNELS)] * (BLOCKS - 1) + [(BITS, CHANNELS)]:
            c = torch.from_numpy(w["conv_w"][at:at + cout * cin * 9].reshape(cout, cin, 3, 3)).cuda()
            self.convs.append(c.permute(2, 3, 1, 0).reshape(9 * cin, cout).contiguous())
            at += cout * cin * 9
        self.lin_w, self.lin_b = (torch.from_numpy(w[k]).cuda() for k in ("lin_w", "lin_b"))

    def __call__(self, images):
        x = (images - self.mean) / self.std
        for w in self.convs[:-1]:
            x = torch.relu(conv3x3(x, w))
        return conv3x3(x, self.convs[-1]).mean(dim=(1, 2)) @ self.lin_w.t() + self.lin_b


def encode(ctx, message):
    """The systematic code word of a message [k] (remainder of its polynomial by the code's generator), checked with the library's decoder."""
    n, k, q = CODE["n"], CODE["k"], 1 << CODE["m"]
    exp, log, x = [0] * (2 * q), [0] * q, 1
    for i in range(q - 1):
        exp[i] = exp[i + q - 1] = x
        log[x] = i
        x <<= 1
        if x & q:
            x ^= CODE["prim_poly"]
    mul = lambda a, b: exp[log[a] + log[b]] if a and b else 0
    gpoly = [1]
    for r in range(CODE["fcr"], CODE["fcr"] + n - k):
        gpoly = [(gpoly[i] if i < len(gpoly) else 0) ^ (mul(gpoly[i - 1], exp[r]) if i else 0) for i in range(len(gpoly) + 1)]
    rest = list(message) + [0] * (n - k)
    for i in range(k):
        lead = rest[i]
        for j, c in enumerate(gpoly):
            rest[i + j] ^= mul(lead, c)
    word = np.array(list(message) + rest[k:], dtype=np.uint8)
    d = torch.from_numpy(word[None]).cuda()
    msg, nerr = torch.empty((1, k), dtype=torch.uint8, device="cuda"), torch.empty(1, dtype=torch.int8, device="cuda")
    ctx.qrm_rs_decode(d, 1, msg, None, nerr)
    assert int(nerr[0]) == 0 and np.array_equal(msg[0].cpu().numpy(), message), "not a code word"
    return word


def detect(ctx, images):
    """The detector on images [N,32,32,3] in 0..1 as 8-bit planes -> bits, corrected symbols, matches, detected."""
    n = images.shape[0]
    planes = (images.detach().clamp(0, 1) * 255).round().to(torch.uint8).permute(0, 3, 1, 2).contiguous()
    empty = lambda shape, t=torch.uint8: torch.empty(shape, dtype=t, device="cuda")
    bits, msg, nerr, matches, found = empty((n, BITS)), empty((n, CODE["k"])), empty((n,), torch.int8), empty((n,), torch.int32), empty((n,))
    ctx.qrm_detect_verify(planes, n, SIDE, SIDE, None, SIDE, None, bits, msg, None, nerr, matches, found)
    torch.cuda.synchronize()
    return bits, nerr, matches, found


def main(steps=200, batch=4, moment_bits=8, peak_lr=5e-3, rs_weight=0.05, fidelity=10.0, seed=0, report=print, attention=False, clip=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    decoder, weights = Decoder(gen, attention), extractor_weights(rng)
    code = qrm.Context(rs=CODE)

    # the extractor's linear layer is made to whiten what the extractor sees in images of this decoder and in noisy ones: every bit then starts as a fair
    # coin that says nothing of the others
    z = torch.randn((256, 16, 16, 8), generator=gen, device="cuda")
    sample = decoder(z, code).detach()
    noise = torch.rand((256, SIDE, SIDE, 3), generator=gen, device="cuda") - 0.5
    sample = torch.cat([sample, (sample + 0.5 * noise).clamp(0, 1), (sample + 0.2 * noise.mean(dim=3, keepdim=True)).clamp(0, 1)])
    weights["lin_w"], weights["lin_b"] = np.eye(BITS, dtype=np.float32), np.zeros(BITS, np.float32)
    pooled = Extractor(weights)(sample).double().cpu().numpy()
    power, axes = np.linalg.eigh(np.cov(pooled.T))
    mix = np.linalg.qr(rng.normal(size=(BITS, BITS)))[0]     # (so that no bit is one axis alone)
    weights["lin_w"] = (mix @ (axes / np.sqrt(power + WHITEN * power.max())).T).astype(np.float32)
    weights["lin_b"] = -(weights["lin_w"] @ pooled.mean(axis=0)).astype(np.float32)
    extractor, ctx = Extractor(weights), qrm.Context(weights=weights, rs=CODE)

    key = rng.integers(0, 1 << CODE["m"], CODE["k"]).astype(np.uint8)
    word = encode(ctx, key)
    target = torch.from_numpy(((word[:, None] >> np.arange(CODE["m"] - 1, -1, -1)) & 1).astype(np.uint8).reshape(-1)).cuda()
    ctx.qrm_set_key(key, qrm.qrm_key_threshold(CODE["k"] * CODE["m"], 1e-6))

    rows = []
    for p in decoder.params:
        n = p.numel()
        row = dict(param=p.detach(), weight_decay=0.01 if p.dim() > 1 else 0.0)
        if moment_bits == 8:
            blocks = -(-n // 256)
            row.update(m=torch.zeros(n, dtype=torch.int8, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                       m_scale=torch.zeros(blocks, device="cuda"), v_scale=torch.zeros(blocks, device="cuda"))
        else:
            row.update(m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"))
        rows.append(row)
    opt = qrm.AdamW(ctx, rows, torch.float32)

    held_out = torch.randn((16, 16, 16, 8), generator=gen, device="cuda")
    before = decoder(held_out, ctx).detach()
    frozen = [p.detach().clone() for p in decoder.params]
    errors, history = torch.empty(batch, dtype=torch.int32, device="cuda"), []
    norm, scale = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    for step in range(1, steps + 1):
        z = torch.randn((batch, 16, 16, 8), generator=gen, device="cuda")
        with torch.no_grad():                                # what the decoder made of these latents before
            kept = [p.detach().clone() for p in decoder.params]
            for p, f in zip(decoder.params, frozen):
                p.copy_(f)
            original = decoder(z, ctx)
            for p, k in zip(decoder.params, kept):
                p.copy_(k)
        images = decoder(z, ctx)
        loss = MessageLoss.apply(extractor(images), target, ctx, rs_weight, errors) + fidelity * (images - original).square().mean()
        grads = torch.autograd.grad(loss, decoder.params)
        warm = min(1.0, step / 20)
        lr = warm * (1e-6 + (peak_lr - 1e-6) * 0.5 * (1 + math.cos(math.pi * max(0, step - 20) / max(1, steps - 20))))
        grads = [g.contiguous() for g in grads]
        if clip > 0.0:
            opt.qrm_adamw_grad_norm(grads, clip, norm, scale)
        opt.qrm_adamw_step(grads, step, lr, d_grad_scale=scale if clip > 0.0 else None)
        history.append(float(loss.detach()))
        if step % 25 == 0 or step == 1:
            report(f"step {step:4d}  loss {history[-1]:.4f}  wrong bits an image {float(errors.float().mean()):.1f} of {BITS}")

    results = {}
    for name, images in (("before", before), ("after", decoder(held_out, ctx))):
        bits, nerr, matches, found = detect(ctx, images)
        wrong = (bits != target).sum(dim=1).float().mean()
        results[name] = dict(wrong=float(wrong), detected=int(found.sum()), images=int(found.numel()), matches=matches.cpu().numpy(), nerr=nerr.cpu().numpy())
        report(f"{name:6s}: {float(wrong):.1f} wrong bits an image before correction, key found in {int(found.sum())} of {found.numel()} images")
    results["change"] = float((decoder(held_out, ctx).detach() - before).square().mean().sqrt())
    report(f"mean change of a pixel {255 * results['change']:.1f} of 255")
    opt.close()
    ctx.close()
    code.close()
    return history, results


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--steps", type=int, default=200)
    a.add_argument("--bits", type=int, default=8, choices=(8, 32), help="of the optimiser's moments")
    a.add_argument("--seed", type=int, default=0)
    a.add_argument("--attention", action="store_true", help="the decoder's pixels look at each other")
    a.add_argument("--clip", type=float, default=0.0, help="bound of the gradients' norm, 0 for none")
    args = a.parse_args()
    main(steps=args.steps, moment_bits=args.bits, seed=args.seed, attention=args.attention, clip=args.clip)
