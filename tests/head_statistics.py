"""How far logits may be off in the root mean square when bf16 products are added up in fp32 on the tensor cores, and what that does to the
numbers made of them.  A worst case over d additions (head_reference) is so wide at real widths that logits rounded to 16 bits pass.

One instruction adds 16 products to the accumulator.  All 17 are cut off at the last place that fp32 has at the size of the largest, 2^-23 of
it at most.  What is cut off the products has their random signs and adds up like a walk, 4 x 0.58 last places (the root mean square of a
number in [0, 1)) if all were as long as the largest, and 0.58 of the accumulator itself, which is the same way in every step: below
2 last places a step where, as here, most products are far smaller than the accumulator.  So a logit is off by at most
    2 x 2^-23 x sum over the steps of max(|sum before|, |sum after|, largest product)
in the root mean square over rows."""
import math

import torch

STEP = 16


def logit_errors(H, W):
    """That sum of every logit, [T, V] in 64 bits, and the logits."""
    h, w = H.double(), W.double()
    s = torch.zeros(len(h), len(w), dtype=torch.float64, device=H.device)
    total = torch.zeros_like(s)
    for k in range(0, h.shape[1], STEP):
        a, b = h[:, k:k + STEP], w[:, k:k + STEP]
        before = s.abs()
        s = s + a @ b.T
        largest = torch.zeros_like(s)
        for i in range(a.shape[1]):
            torch.maximum(largest, a[:, i:i + 1].abs() * b[:, i].abs(), out=largest)
        total += torch.maximum(torch.maximum(before, s.abs()), largest)
    return 2 * 2.0 ** -23 * total, s


def bounds(H, W, y, mask, smooth, z_coef):
    """dict of (value, bound) per row that counts, and of the loss."""
    on = mask.bool()
    e, z = logit_errors(H[on], W)
    T, V = z.shape
    y = y[on].long()[:, None]
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    zy, zbar = z.gather(1, y)[:, 0], z.mean(1)
    # exponentials to 2^-21, their arguments and the logarithm to a few last places of lse and log V
    dlse = (p * e).sum(1) + 2.0 ** -21 + 2.0 ** -22 * (lse.abs() + math.log(V))
    dlogp = e.gather(1, y)[:, 0] + dlse
    # the mean logit is a sum of V numbers in fp32
    dbar = e.mean(1) + V * 2.0 ** -24 * z.abs().mean(1)
    each = (1 - smooth) * (lse - zy) + smooth * (lse - zbar) + z_coef * lse ** 2
    deach = (1 - smooth) * dlogp + smooth * (dlse + dbar) + 2 * z_coef * lse.abs() * dlse + 2.0 ** -22 * (each.abs() + lse.abs())
    return dict(logp=(zy - lse, dlogp), lse=(lse, dlse), token_loss=(each, deach), loss=(each.mean().reshape(1), deach.mean().reshape(1)))


def assert_within_in_the_mean(got, want, bound, what):
    rms = lambda x: x.double().square().mean().sqrt().item()  # noqa: E731
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    assert rms(got.double() - want) <= rms(bound), f"{what}: off by {rms(got.double() - want):.2e}, at most {rms(bound):.2e}"
