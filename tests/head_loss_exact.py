"""The losses on top of the head in float64 on the device, with how far a kernel's gradients may be off, element
by element.

Bars. A logit is a sum of H products in float32: each of the H / 16 matrix instructions of a K loop (six times as
many where a float32 product is split) rounds the running sum, which stays below the largest logit z, by at most
2^-23 of it, so a logit is off by at most eps = H / 16 (x 6) x 2^-23 x max |z|, and an exponential or a probability p
by twice that of itself (the log-sum-exp is off as well), and 1e-5 for exponentials, logarithms and sums. A gradient
G = sum dz x, dz = c (a p - b q), x rows of W or H, is then off by at most
    (2 eps + 1e-5) sum c (a p + b q) |x|,
for bf16 operands also by what rounding the exponentials to 11 bits and dz to 8 gives, (2^-11 + 2^-8) sum |dz| |x|, and
by the output's own rounding, 2^-8 |G| (2^-23 for float32)."""
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def head_loss(h, w, c, target=None, ids=None, teacher=None, tau=1.0, z_coef=0.0):
    """Cross entropy of `target`, or distillation from `teacher` logits at `ids` (-1: none), with factors c [T] (0 where
    the mask is 0). dict(token, lse, dhidden, dw, and for either gradient the two sums of the bar)."""
    hd, wd, c = h.double(), w.double(), c.double()[:, None]
    z = hd @ wd.t() / tau
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - lse)
    on = (c != 0).double()
    q = torch.zeros_like(z)
    if target is not None:
        q.scatter_(1, target.long()[:, None], 1.0)
        token = lse - z.gather(1, target.long()[:, None])
        a = 1.0 + 2.0 * z_coef * lse
    else:
        u = torch.where(ids >= 0, teacher.double() / tau, -torch.inf)
        some = (u > -torch.inf).any(1, keepdim=True)   # a row without an entry: q = 0
        logq = torch.where(some, torch.log_softmax(u, 1), -torch.inf)
        qk = torch.exp(logq)
        at = ids.long().clamp(min=0)
        q.scatter_add_(1, at, qk)
        token = tau ** 2 * torch.where(qk > 0, qk * (logq - z.gather(1, at) + lse), 0.0).sum(1, keepdim=True)
        a = qk.sum(1, keepdim=True)
    out = dict(token=(token * on)[:, 0], lse=(lse * on)[:, 0], z=float(z.abs().max()))
    dz = c * tau * (a * p - q)
    both = c * tau * (a * p + q)
    out["dhidden"], out["dw"] = dz @ wd, dz.t() @ hd
    out["dhidden_rounded"], out["dw_rounded"] = dz.abs() @ wd.abs(), dz.abs().t() @ hd.abs()
    out["dhidden_both"], out["dw_both"] = both @ wd.abs(), both.t() @ hd.abs()
    return out


def logit_eps(H, z, dtype):
    return H / 16 * (6 if dtype == "f32" else 1) * 2.0 ** -23 * z


def grad_bar(ref, name, H, dtype, out_bits=None):
    """Elementwise bar of gradient `name`; out_bits: significand bits it is stored with (24, 8)."""
    bar = (2 * logit_eps(H, ref["z"], dtype) + 1e-5) * ref[name + "_both"]
    if dtype == "bf16":
        bar = bar + (2.0 ** -11 + 2.0 ** -8) * ref[name + "_rounded"]
    bits = out_bits or {"f32": 24, "bf16": 8}[dtype]
    return bar + 2.0 ** (-bits if bits < 24 else -23) * ref[name].abs()


def check_grad(got, ref, name, H, dtype, out_bits=None):
    assert torch.isfinite(got).all(), name
    over = (got.double() - ref[name]).abs() - grad_bar(ref, name, H, dtype, out_bits)
    worst = int(over.argmax())
    assert float(over.max()) <= 0.0, (name, divmod(worst, got.shape[1]), float(got.reshape(-1)[worst]),
                                      float(ref[name].reshape(-1)[worst]))
