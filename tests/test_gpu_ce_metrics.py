"""Every number of the supervised loss's report against its definition in 64 bits, on the paths that add it up differently."""
import pytest
import torch

from tests.head_reference import assert_within, cross_entropy

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _inputs(T, d, V, seed):
    """Targets that are their row's largest logit or its smallest, by more than any sum in fp32 can be off.  What all rows share moves the
    mean logit away from zero, or `lse - mean z` and `lse` were the same number."""
    g = torch.Generator(DEV).manual_seed(seed)
    W = (torch.randn(V, d, generator=g, device=DEV) * 0.05 + 0.01).bfloat16()
    H = (torch.randn(T, d, generator=g, device=DEV) + 0.5).bfloat16()
    mask = (torch.rand(T, generator=g, device=DEV) < 0.7).to(torch.uint8)
    z = H.double() @ W.double().T
    dz = (H.double().abs() @ W.double().abs().T).amax(1) * d * 2.0 ** -23
    top, at = z.topk(2, 1)
    largest = (top[:, 0] - top[:, 1] > 4 * dz) & (torch.rand(T, generator=g, device=DEV) < 0.6)
    y = torch.where(largest, at[:, 0], z.argmin(1)).int()
    assert bool((z.amax(1) - z.amin(1) > 4 * dz).all())
    return H, W, y, mask, z, dz


def _metrics(H, y, mask, z, dz, ref, weight):
    """Values, and how far sums and roundings in fp32 may move them."""
    V = z.shape[1]
    on = mask.bool()
    wt = on.double() / on.sum() if weight is None else torch.where(on, weight.double(), 0.0)
    lse = torch.logsumexp(z, 1)
    zy, zbar = z.gather(1, y.long()[:, None])[:, 0], z.mean(1)
    dlse = dz + 1e-6 * (lse.abs() + 12)
    # a mean logit: every logit's error, and V additions in fp32 in whatever order
    dbar = dz + V * 2.0 ** -24 * z.abs().mean(1)
    rows = [(lse - zy, dz + dlse), (lse - zbar, dlse + dbar), (lse ** 2, 2 * lse.abs() * dlse + dlse ** 2),
            ((zy >= z.amax(1)).double(), torch.zeros_like(lse)), (lse, dlse)]
    # the token mean's weight and a row's number are rounded once each, their products are added up in 64 bits
    value = [(wt * v).sum() for v, _ in rows] + [torch.where(on, lse - zy, 0.0).max()]
    bound = [(wt.abs() * (b + 2.0 ** -22 * v.abs())).sum() for v, b in rows] + [torch.where(on, dz + dlse, 0.0).max()]
    value, bound = torch.stack(value), torch.stack(bound)
    if weight is None:
        assert (value - ref["metrics"]).abs().max().item() <= 1e-9 * (1 + value.abs().max().item())
    return value, bound


@pytest.mark.parametrize("T,d,V", [(5, 64, 40), (300, 192, 1500), (300, 960, 1500), (700, 1024, 1800)])
@pytest.mark.parametrize("limits", [(0, 0), (128, 0), (128, 512)])
@pytest.mark.parametrize("weighted", [False, True])
def test_all_of_the_report(T, d, V, limits, weighted):
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        c.set_slab_limits(*limits)
        H, W, y, mask, z, dz = _inputs(T, d, V, T + d)
        mask[:3] = torch.tensor([1, 0, 1], dtype=torch.uint8)
        weight = torch.rand(T, generator=torch.Generator(DEV).manual_seed(1), device=DEV) / 100 - 0.001 if weighted else None   # some below zero
        ref = cross_entropy(H, W, y, mask, 0.1, 1e-3, weight)
        value, bound = _metrics(H, y, mask, z, dz, ref, weight)
        # numbers in each other's places would show
        apart = (value[:, None] - value).abs() - (bound[:, None] + bound) + torch.eye(6, device=DEV) * 1e9
        assert T < 100 or apart.min().item() > 0
        for kw in (dict(), dict(dW_bf16=True), dict(want_dH=False), dict(want_dH=False, want_dW=False)):
            out = c.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1, z_coef=1e-3, token_weight=weight, **kw)
            assert c.last_device_status()[0] == 0
            assert_within(out["metrics"][:6], value, bound, "metrics")
            assert out["metrics"][6].item() == int(mask.sum()) and out["metrics"][7].item() == 0
    finally:
        c.close()


def test_a_report_of_nothing():
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        H, W, y, mask, _, _ = _inputs(20, 64, 30, 3)
        for rows in (20, 0):
            out = c.rl_cross_entropy_fwd_bwd(H[:rows], W, y[:rows], torch.zeros_like(mask[:rows]))
            assert bool((out["metrics"] == 0).all())
    finally:
        c.close()
