"""Definitions in 64 bits that the tests of the supervised loss and of the 8-bit head compare with, and what fp32 sums and bf16
roundings may move (torch.float64 on whatever device the inputs are)."""
import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def quantize_rows(x):
    """q, scale of rows, from the definition: r = fl(127 / m), s = fl(m / 127), q = rint(x r)."""
    x64 = x.double()
    m = x64.abs().amax(1)
    bad, small = ~torch.isfinite(x64).all(1), m < 2.0 ** -100
    m = torch.where(bad | small, torch.ones_like(m), m)
    r, s = (torch.full_like(m, 127) / m).float().double(), (m / torch.full_like(m, 127)).float()
    q = torch.round(torch.where(bad[:, None], torch.zeros_like(x64), x64) * r[:, None])
    q[bad | small] = 0
    s[small] = 0.0
    s[bad] = float("nan")
    return q, s


def cross_entropy(H, W, y, mask=None, smooth=0.0, z_coef=0.0, weight=None, count=None):
    """Everything rl_cross_entropy_fwd_bwd returns, and bounds on how far fp32 sums and G in bf16 may be off: dict of (value, bound)."""
    T, d = H.shape
    V = W.shape[0]
    mask = torch.ones(T, dtype=torch.bool, device=H.device) if mask is None else mask.bool()
    h, w = torch.where(mask[:, None], H.double(), 0.0), W.double()
    y = torch.where(mask, y.long(), 0)
    n = int(mask.sum()) if count is None else count
    wt = mask.double() / max(n, 1) if weight is None else torch.where(mask, weight.double(), 0.0)
    z = h @ w.T
    # a sum of d products in fp32, in any order and with truncated additions: d steps of 2^-23 of the sum of magnitudes
    dz = (h.abs() @ w.abs().T).amax(1) * d * 2.0 ** -23
    lse = torch.logsumexp(z, 1)
    zy, zbar = z.gather(1, y[:, None])[:, 0], z.mean(1)
    each = (1 - smooth) * (lse - zy) + smooth * (lse - zbar) + z_coef * lse ** 2
    # exponentials to 2^-21, their sums and logarithm to a few 2^-24 of values up to |lse| and log V
    dlse = dz + 1e-6 * (lse.abs() + 12)
    deach = 2 * dlse + 2 * z_coef * lse.abs() * dlse + 1e-6 * (each.abs() + zbar.abs() + 1) * (1 + smooth * 8)
    p = torch.exp(z - lse[:, None])
    G = wt[:, None] * (1 + 2 * z_coef * lse)[:, None] * p - (wt * smooth / V)[:, None]
    G[torch.arange(T, device=H.device), y] -= wt * (1 - smooth)
    # before its rounding G is off by p's error and by a few 2^-24 of the terms it is the difference of
    size = wt.abs()
    terms = size[:, None] * (1 + 2 * z_coef * lse.abs())[:, None] * p
    dG = terms * (dz + dlse + 4e-6)[:, None] + 2.0 ** -8 * G.abs() + 2.0 ** -22 * (terms + (size * smooth / V)[:, None])
    dG[torch.arange(T, device=H.device), y] += 2.0 ** -22 * size * (1 - smooth)
    aG = G.abs() + dG
    dH, dW = G @ w, G.T @ h
    ddH = dG @ w.abs() + (aG @ w.abs()) * V * 2.0 ** -23
    ddW = dG.T @ h.abs() + (aG.T @ h.abs()) * T * 2.0 ** -23
    zero = lambda x: torch.where(mask, x, 0.0)  # noqa: E731
    return dict(loss=((wt * each).sum(), (wt.abs() * deach).sum() + 2.0 ** -23 * (wt * each).abs().sum()),
                logp=(zero(zy - lse), zero(dz + dlse)), lse=(zero(lse), zero(dlse)), token_loss=(zero(each), zero(deach)),
                dH=(dH, ddH), dW=(dW, ddW), G=(G, dG),
                metrics=torch.stack([(wt * (lse - zy)).sum(), (wt * (lse - zbar)).sum(), (wt * lse ** 2).sum(),
                                     (wt * (zy >= z.amax(1)).double()).sum(), (wt * lse).sum(), zero(lse - zy).max()]))


def assert_within(got, want, bound, what):
    """|got - want| <= bound + what rounding to got's type moves, everywhere."""
    over = (got.double() - want).abs() - (bound + HALF_STEP[got.dtype] * (want.abs() + bound) + 1e-30)
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    assert over.numel() == 0 or over.max().item() <= 0, f"{what}: {over.max().item():.3e} over its bound at {int(over.argmax())}"
