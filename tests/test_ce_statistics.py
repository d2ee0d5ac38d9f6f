"""logp, lse and losses at real widths, in the root mean square: close enough that logits held in 16 bits anywhere would show."""
import pytest
import torch

from tests.head_statistics import assert_within_in_the_mean, bounds

WIDTHS = [896, 1024, 2048, 3584]
SMOOTH, Z_COEF = 0.1, 1e-3


def _inputs(T, d, V, device, seed=0):
    g = torch.Generator(device).manual_seed(seed + d)
    std = 0.05
    W = (torch.randn(V, d, generator=g, device=device) * std).bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device=device, dtype=torch.int32)
    sure = torch.rand(T, generator=g, device=device) * 8 / (std * std * d)
    H = (torch.randn(T, d, generator=g, device=device) + sure[:, None] * W[y.long()].float()).bfloat16()
    mask = (torch.rand(T, generator=g, device=device) < 0.8).to(torch.uint8)
    return H, W, y, mask


def _numbers(z, y, mask):
    on = mask.bool()
    z, y = z.double()[on], y[on].long()[:, None]
    lse, zy = torch.logsumexp(z, 1), z.gather(1, y)[:, 0]
    each = (1 - SMOOTH) * (lse - zy) + SMOOTH * (lse - z.mean(1)) + Z_COEF * lse ** 2
    return dict(logp=zy - lse, lse=lse, token_loss=each, loss=each.mean().reshape(1))


@pytest.mark.parametrize("d", WIDTHS)
def test_the_bounds_tell_fp32_logits_from_16_bit_ones(d):
    H, W, y, mask = _inputs(48, d, 700, "cpu")
    want = bounds(H, W, y, mask, SMOOTH, Z_COEF)
    z = H.float() @ W.float().T
    for key, x in _numbers(z, y, mask).items():
        assert_within_in_the_mean(x, *want[key], key)
    for kind in (torch.float16, torch.bfloat16):
        got = _numbers(z.to(kind), y, mask)
        for key in ("logp", "lse", "token_loss"):
            with pytest.raises(AssertionError):
                assert_within_in_the_mean(got[key], *want[key], key)
    # inputs rounded to the 11 bits that the tensor cores' shorter formats keep
    got = _numbers((z.double() * (1 + 2.0 ** -11)), y, mask)
    for key in ("logp", "lse", "token_loss"):
        with pytest.raises(AssertionError):
            assert_within_in_the_mean(got[key], *want[key], key)


@pytest.mark.gpu
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("limits", [(0, 0), (128, 0), (256, 512)])   # slabs of whole rows keep their logits, slabs of columns form them twice
def test_statistics_of_the_supervised_loss(d, limits):
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        c.set_slab_limits(*limits)
        H, W, y, mask = _inputs(400, d, 1300, "cuda:0")
        on = mask.bool()
        want = bounds(H, W, y, mask, SMOOTH, Z_COEF)
        for kw in (dict(), dict(dW_bf16=True, want_dH=False), dict(want_dW=False), dict(want_dH=False, want_dW=False)):
            out = c.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=SMOOTH, z_coef=Z_COEF, **kw)
            assert c.last_device_status()[0] == 0
            for key in ("logp", "lse", "token_loss"):
                assert_within_in_the_mean(out[key][on], *want[key], key)
            assert_within_in_the_mean(out["loss"], *want["loss"], "loss")
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1024, 2048])
def test_statistics_over_a_whole_vocabulary(d):
    """Many column ranges a row, merged at the end."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        H, W, y, mask = _inputs(64, d, 50257, "cuda:0")
        on = mask.bool()
        want = bounds(H, W, y, mask, 0.0, Z_COEF)
        for kw in (dict(dW_bf16=True), dict(want_dH=False, want_dW=False)):
            out = c.rl_cross_entropy_fwd_bwd(H, W, y, mask, z_coef=Z_COEF, **kw)
            for key in ("logp", "lse", "token_loss"):
                assert_within_in_the_mean(out[key][on], *want[key], key)
            assert_within_in_the_mean(out["loss"], *want["loss"], "loss")
    finally:
        c.close()
