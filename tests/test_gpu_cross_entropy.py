"""The supervised loss on the head against its definition in 64 bits, within what fp32 sums and a bf16 gradient of the logits may move
(head_reference), on every path the call takes: narrow and wide heads, slabs of rows and of columns, one or both gradients, none."""
import numpy as np
import pytest
import torch

from tests.head_reference import assert_within, cross_entropy, quantize_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_21450_b200 import Context
    c = Context(0)
    yield c
    c.close()


def _inputs(T, d, V, seed=0, masked=0.0, std=0.05, sure=8.0):
    g = torch.Generator(DEV).manual_seed(seed)
    W = (torch.randn(V, d, generator=g, device=DEV) * std).bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    a = torch.rand(T, generator=g, device=DEV) * sure / (std * std * d)
    H = (torch.randn(T, d, generator=g, device=DEV) + a[:, None] * W[y.long()].float()).bfloat16()
    mask = (torch.rand(T, generator=g, device=DEV) >= masked).to(torch.uint8) if masked else None
    return H, W, y, mask


def _check(ctx, H, W, y, mask, ref_H=None, **kw):
    """One call on poisoned outputs against the definition."""
    T, d = H.shape
    V = W.shape[0]
    bf16, fp32 = kw.get("dW_bf16", False), kw.get("dH_fp32", False)
    dH = torch.full((T, d), float("nan"), dtype=torch.float32 if fp32 else torch.bfloat16, device=DEV)
    dW = torch.full((V, d), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
    out = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, dH=dH, dW=dW, **kw)
    s, detail = ctx.last_device_status()
    assert s == 0, (s, hex(detail))
    ref = cross_entropy(H if ref_H is None else ref_H, W, y, mask, kw.get("label_smoothing", 0.0), kw.get("z_coef", 0.0),
                        kw.get("token_weight"))
    assert ("dH" in out) == kw.get("want_dH", True) and ("dW" in out) == kw.get("want_dW", True)
    for key in ("loss", "logp", "lse", "token_loss", "dH", "dW"):
        if key in out:
            want, bound = ref[key]
            assert_within(out[key], want.reshape(out[key].shape), bound.reshape(out[key].shape), key)
    n = T if mask is None else int((mask != 0).sum())
    m = out["metrics"].double()
    assert m[6].item() == n and abs(m[0].item() - ref["metrics"][0].item()) <= ref["logp"][1].max().item() * max(1.0, ref["loss"][1].item()) + 1e-6 * abs(m[0].item())
    if mask is not None:
        off = mask == 0
        for key in ("logp", "lse", "token_loss", "dH"):
            if key in out:
                assert bool((out[key][off] == 0).all()), key
    return out, ref


SHAPES = [(1, 64, 1), (1, 64, 2), (2, 64, 255), (5, 128, 257), (130, 192, 1000), (256, 256, 4096), (77, 896, 2049), (300, 1024, 1537),
          (129, 960, 512), (640, 2048, 1300), (1025, 1088, 777)]


@pytest.mark.parametrize("T,d,V", SHAPES)
@pytest.mark.parametrize("smooth,z_coef", [(0.0, 0.0), (0.1, 1e-3)])
def test_against_definition(ctx, T, d, V, smooth, z_coef):
    H, W, y, mask = _inputs(T, d, V, seed=T + d + V, masked=0.3 if T > 4 else 0.0)
    _check(ctx, H, W, y, mask, label_smoothing=smooth, z_coef=z_coef)
    _check(ctx, H, W, y, mask, label_smoothing=smooth, z_coef=z_coef, dW_bf16=True, dH_fp32=True)


@pytest.mark.parametrize("T,d,V", [(5, 128, 257), (256, 256, 4096), (300, 1024, 1537)])
def test_one_gradient_or_none(ctx, T, d, V):
    H, W, y, mask = _inputs(T, d, V, seed=3, masked=0.2)
    kw = dict(label_smoothing=0.05, z_coef=1e-4)
    both, _ = _check(ctx, H, W, y, mask, **kw)
    for more in (dict(want_dW=False), dict(want_dH=False), dict(want_dH=False, dW_bf16=True), dict(want_dH=False, want_dW=False)):
        out, _ = _check(ctx, H, W, y, mask, **kw, **more)
        for key in ("logp", "lse", "loss"):
            assert torch.allclose(out[key], both[key], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("limits", [(128, 0), (0, 256), (256, 512), (128, 8192)])
@pytest.mark.parametrize("d", [192, 960])
def test_slabs(limits, d):
    """Rows and columns of the gradient in several slabs; a bf16 dW is then added up in fp32."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        c.set_slab_limits(*limits)
        H, W, y, mask = _inputs(700, d, 1800, seed=9, masked=0.25)
        for kw in (dict(), dict(dW_bf16=True), dict(want_dW=False), dict(want_dH=False), dict(want_dH=False, dW_bf16=True)):
            _check(c, H, W, y, mask, label_smoothing=0.1, z_coef=1e-3, **kw)
        few = torch.zeros(700, dtype=torch.uint8, device=DEV)
        few[650:660] = 1                                            # slabs sized for 700 rows, ten that count
        _check(c, H, W, y, few, dW_bf16=True)
    finally:
        c.close()


@pytest.mark.parametrize("T,d,V", [(1000, 1024, 151936), (1500, 2048, 100001)])
def test_gradient_formed_by_the_dH_launch(ctx, T, d, V):
    """Large enough (T * V) for dH to form its operand itself, with and without dW behind it."""
    H, W, y, mask = _inputs(T, d, V, seed=21, masked=0.1, std=0.02)
    for kw in (dict(dW_bf16=True), dict(want_dW=False)):
        out = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1, z_coef=1e-4, **kw)
        assert ctx.last_device_status()[0] == 0
        ref = cross_entropy(H, W, y, mask, 0.1, 1e-4)
        for key in ("loss", "logp", "dH"):
            want, bound = ref[key]
            assert_within(out[key], want.reshape(out[key].shape), bound.reshape(out[key].shape), key)
        rel = lambda k: ((out[k].double() - ref[k][0]).norm() / ref[k][0].norm()).item()  # noqa: E731
        # every G is off by 2^-8 at most, independently, the result by half a step: 2^-8 in all is generous
        assert rel("dH") <= 2.0 ** -8 and ("dW" not in out or rel("dW") <= 2.0 ** -8)


def test_differences():
    """dH and dW against differences of the loss's definition along random directions."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        H, W, y, mask = _inputs(60, 128, 300, seed=5, masked=0.3)
        out = c.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1, z_coef=1e-2, dH_fp32=True)
        g = torch.Generator(DEV).manual_seed(1)
        loss = lambda h, w: cross_entropy(h, w, y, mask, 0.1, 1e-2)["loss"][0]  # noqa: E731
        ref = cross_entropy(H, W, y, mask, 0.1, 1e-2)
        for x, key in ((H, "dH"), (W, "dW")):
            u = torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
            e = 1e-5
            hi, lo = ((x.double() + t * u) for t in (e, -e))
            diff = (loss(hi, W) - loss(lo, W)) / (2 * e) if key == "dH" else (loss(H, hi) - loss(H, lo)) / (2 * e)
            got = (out[key].double() * u).sum()
            assert abs((got - diff).item()) <= (ref[key][1] * u.abs()).sum().item() + 1e-8 * (1 + abs(diff.item()))
    finally:
        c.close()


def test_masked_rows_may_hold_anything(ctx):
    H, W, y, mask = _inputs(200, 256, 500, seed=8, masked=0.4)
    off = mask == 0
    clean = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1)
    H2, y2 = H.clone(), y.clone()
    H2[off] = float("nan")
    H2[off.nonzero()[:3, 0]] = float("inf")
    y2[off] = torch.randint(-2 ** 31, 2 ** 31 - 1, (int(off.sum()),), dtype=torch.int32, device=DEV)
    out = ctx.rl_cross_entropy_fwd_bwd(H2, W, y2, mask, label_smoothing=0.1)
    assert ctx.last_device_status()[0] == 0
    for k in clean:
        assert torch.equal(out[k], clean[k]), k


def test_nothing_that_counts(ctx):
    H, W, y, _ = _inputs(100, 256, 300)
    none = torch.zeros(100, dtype=torch.uint8, device=DEV)
    for bf16 in (False, True):
        dW = torch.full((300, 256), 7.0, dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV)
        out = ctx.rl_cross_entropy_fwd_bwd(H, W, y, none, label_smoothing=0.1, z_coef=1.0, dW_bf16=bf16, dW=dW)
        for k in ("loss", "dH", "dW", "logp", "lse", "token_loss"):
            assert bool((out[k] == 0).all()), k
        dW.fill_(7.0)
        out = ctx.rl_cross_entropy_fwd_bwd(H[:0], W, y[:0], None, dW_bf16=bf16, dW=dW)
        assert out["loss"].item() == 0 and bool((dW == 0).all()) and out["dH"].shape == (0, 256)
    out = ctx.rl_cross_entropy_fwd_bwd(H, W, y, none, want_dH=False, want_dW=False)
    assert out["loss"].item() == 0
    kept = torch.full((300, 256), 7.0, device=DEV)
    ctx.rl_cross_entropy_fwd_bwd(H[:0], W, y[:0], None, accumulate_dW=True, dW=kept)
    assert bool((kept == 7).all())


def test_weights_count_and_accumulation(ctx):
    H, W, y, mask = _inputs(150, 960, 700, seed=2, masked=0.3)
    wt = torch.rand(150, device=DEV) / 50 - 0.002                    # some below zero
    out, ref = _check(ctx, H, W, y, mask, token_weight=wt, label_smoothing=0.1)
    count = torch.tensor([400], dtype=torch.int64, device=DEV)
    got = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, token_count=count)
    want = cross_entropy(H, W, y, mask, count=400)
    assert_within(got["loss"], want["loss"][0].reshape(1), want["loss"][1].reshape(1), "loss")
    assert_within(got["dW"], *want["dW"], "dW")
    one = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask)["dW"].clone()
    twice = one.clone()
    ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, accumulate_dW=True, dW=twice)
    assert (twice - 2 * one).abs().max().item() <= 2.0 ** -22 * one.abs().max().item()


def test_agrees_with_the_policy_loss(ctx):
    """The gradient of -mean logp is that of the policy loss with advantage one, old = current log-probabilities and no KL term."""
    H, W, y, mask = _inputs(300, 1024, 3000, seed=4, masked=0.2)
    ce = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask)
    logp = ctx.rl_token_logprobs(H, W, y, mask)[0]
    one = torch.ones(300, device=DEV)
    pl = ctx.rl_policy_loss_fwd_bwd(H, W, y, logp, None, one, mask, 0.2, 0.2, 0.0)
    rel = lambda a, b: ((a.double() - b.double()).norm() / b.double().norm()).item()  # noqa: E731
    # the same G up to the ratio's error (1e-6) before both round it: 2^-8 where that turns a rounding over
    assert rel(ce["dH"], pl["dH"]) <= 2.0 ** -8 and rel(ce["dW"], pl["dW"]) <= 2.0 ** -8
    assert torch.allclose(ce["logp"], pl["logp"], atol=1e-5)


@pytest.mark.parametrize("T,d,V", [(1, 64, 33), (200, 256, 1000), (333, 1024, 1500)])
def test_states_stored_in_8_bits(ctx, T, d, V):
    H, W, y, mask = _inputs(T, d, V, seed=6, masked=0.3 if T > 1 else 0.0)
    Q, scale = ctx.rl_quantize_rows(H)
    q, s = quantize_rows(H)
    assert torch.equal(Q.double(), q) and torch.equal(scale, s)
    stands_for = (q.float() * s[:, None]).bfloat16()                  # both exact in fp32 before the rounding to bf16
    _check(ctx, Q, W, y, mask, ref_H=stands_for, H_scale=scale, label_smoothing=0.1, z_coef=1e-3, dW_bf16=True)
    same = ctx.rl_cross_entropy_fwd_bwd(stands_for, W, y, mask, label_smoothing=0.1)
    out = ctx.rl_cross_entropy_fwd_bwd(Q, W, y, mask, H_scale=scale, label_smoothing=0.1)
    for k in same:
        assert torch.equal(out[k], same[k]), k
    # wider rows, of which a part is taken
    wide = torch.full((T, d + 48), -77, dtype=torch.int8, device=DEV)
    wide[:, :d] = Q
    part = ctx.rl_cross_entropy_fwd_bwd(wide[:, :d], W, y, mask, H_scale=scale, label_smoothing=0.1)
    assert torch.equal(part["dW"], same["dW"])


def test_many_rows_take_the_other_row_map(ctx):
    """More than 32768 rows are counted by launches of their own."""
    T = 33001
    H, W, y, mask = _inputs(T, 64, 50, seed=1, masked=0.5)
    _check(ctx, H, W, y, mask, label_smoothing=0.1)
    Q, scale = ctx.rl_quantize_rows(H)
    _check(ctx, Q, W, y, mask, ref_H=(Q.float() * scale[:, None]).bfloat16(), H_scale=scale)


def test_strided_rows_and_another_stream(ctx):
    H, W, y, mask = _inputs(120, 192, 400, seed=12, masked=0.2)
    want = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask)
    Hs = torch.full((120, 256), float("nan"), dtype=torch.bfloat16, device=DEV)
    Ws = torch.full((400, 200), float("nan"), dtype=torch.bfloat16, device=DEV)
    Hs[:, :192], Ws[:, :192] = H, W
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.rl_cross_entropy_fwd_bwd(Hs[:, :192], Ws[:, :192], y, mask)
    side.synchronize()
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_captured_and_replayed(ctx):
    H, W, y, mask = _inputs(200, 256, 1000, seed=13, masked=0.2)
    dH, dW, loss = torch.empty_like(H), torch.empty_like(W), torch.empty(1, device=DEV)
    call = lambda: ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1, dH=dH, dW=dW, loss=loss, dW_bf16=True)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    H2, _, y2, mask2 = _inputs(200, 256, 1000, seed=14, masked=0.3)
    H.copy_(H2), y.copy_(y2), mask.copy_(mask2)
    graph.replay()
    torch.cuda.synchronize()
    got = dH.clone(), dW.clone(), loss.clone()
    want = ctx.rl_cross_entropy_fwd_bwd(H2, W, y2, mask2, label_smoothing=0.1, dW_bf16=True)
    for a, k in zip(got, ("dH", "dW", "loss")):
        assert torch.equal(a, want[k]), k


@pytest.mark.parametrize("limits", [(0, 0), (128, 0), (128, 512)])
def test_accumulation_and_reports_over_slabs(limits):
    """dW added to over several slabs, and its rows reported while the backward pass runs."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        c.set_slab_limits(*limits)
        H, W, y, mask = _inputs(500, 960, 1300, seed=31, masked=0.3)
        kw = dict(label_smoothing=0.1, z_coef=1e-3)
        want, bound = cross_entropy(H, W, y, mask, 0.1, 1e-3)["dW"]
        start = torch.randn(1300, 960, device=DEV) * 1e-3
        dW = start.clone()
        c.rl_cross_entropy_fwd_bwd(H, W, y, mask, accumulate_dW=True, dW=dW, **kw)
        assert_within(dW, start.double() + want, bound + 2.0 ** -22 * (start.double().abs() + want.abs()), "dW")
        seen = []
        c.set_dw_slab_hook(lambda slab, a, b: seen.append((slab, a, b)))
        got = c.rl_cross_entropy_fwd_bwd(H, W, y, mask, **kw)
        assert [s for s, _, _ in seen] == list(range(len(seen))) and seen[0][1] == 0 and seen[-1][2] == 1300
        assert all(a[2] == b[1] for a, b in zip(seen, seen[1:]))
        assert_within(got["dW"], want, bound, "dW")
        dW = start.clone()
        c.rl_cross_entropy_fwd_bwd(H, W, y, mask, accumulate_dW=True, dW=dW, **kw)
        assert_within(dW, start.double() + want, bound + 2.0 ** -22 * (start.double().abs() + want.abs()), "dW")
    finally:
        c.set_dw_slab_hook(None)
        c.close()


@pytest.mark.parametrize("options", [dict(cta_group=1), dict(wide_tiles=0), dict(dh_stream_k=1), dict(dh_k_slices=3), dict(max_ctas=6),
                                     dict(row_group_bytes=1 << 20)])
def test_options_of_the_context(options):
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        for name, value in options.items():
            getattr(c, "set_" + name)(value)
        H, W, y, mask = _inputs(600, 1024, 2100, seed=32, masked=0.2)
        _check(c, H, W, y, mask, label_smoothing=0.1, z_coef=1e-3, dW_bf16=True)
        _check(c, H, W, y, mask)
        Wq, ws = c.rl_quantize_rows(W)
        for T in (3, 90, 600):
            q, s = c.rl_quantize_rows(H[:T])
            z = (q.double() @ Wq.double().T).float() * s[:, None] * ws
            assert torch.equal(c.rl_int8_linear(H[:T], Wq, ws, out_dtype=torch.float32), z)
            lse = c.rl_token_logprobs_int8(H[:T], Wq, ws, y[:T])[2]
            assert (lse - torch.logsumexp(z.double(), 1)).abs().max().item() <= 1e-6 * (lse.abs().max().item() + 12)
    finally:
        c.close()


def test_between_calls_of_the_policy_loss(ctx):
    """Calls of one context that share its workspace, in turn."""
    H, W, y, mask = _inputs(300, 1024, 3000, seed=33, masked=0.2)
    Wq, ws = ctx.rl_quantize_rows(W)
    old, adv = torch.randn(300, device=DEV) - 8, torch.randn(300, device=DEV)
    policy = lambda: ctx.rl_policy_loss_fwd_bwd(H, W, y, old, old, adv, mask, 0.2, 0.2, 0.04, ent_coef=1e-3)  # noqa: E731
    others = (lambda: ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1, dW_bf16=True),
              lambda: dict(zip("abc", ctx.rl_token_logprobs_int8(H, Wq, ws, y, mask))), lambda: dict(a=ctx.rl_int8_linear(H, Wq, ws)),
              lambda: dict(zip("abc", ctx.rl_token_logprobs(H, W, y, mask))))
    want_policy, want = policy(), [f() for f in others]
    for f, w in zip(others, want):
        for _ in range(2):
            got = f()
            assert all(torch.equal(got[k], w[k]) for k in w)
            got = policy()
            assert all(torch.equal(got[k], want_policy[k]) for k in want_policy)


@pytest.mark.parametrize("limits,T,d,V", [((128, 0), 700, 960, 1800), ((256, 512), 700, 192, 1800), ((0, 0), 500, 1024, 2000), ((128, 0), 3000, 2048, 600),
                                          ((0, 0), 8000, 1024, 151936)])
def test_bf16_dW_is_the_fp32_one_rounded(limits, T, d, V):
    """However many slabs it is added up over."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        c.set_slab_limits(*limits)
        H, W, y, mask = _inputs(T, d, V, seed=35, masked=0.1, std=0.02)
        for m in (mask, torch.cat([mask[:T // 3], torch.zeros_like(mask[T // 3:])])):     # the last slabs have rows, or none
            a = c.rl_cross_entropy_fwd_bwd(H, W, y, m, label_smoothing=0.1, z_coef=1e-4)["dW"].bfloat16()
            for want_dH in (True, False):
                b = c.rl_cross_entropy_fwd_bwd(H, W, y, m, label_smoothing=0.1, z_coef=1e-4, dW_bf16=True, want_dH=want_dH)["dW"]
                assert torch.equal(a, b)
            assert c.last_device_status()[0] == 0
    finally:
        c.close()


def test_twice_the_same(ctx):
    H, W, y, mask = _inputs(700, 2048, 5000, seed=34, masked=0.3)
    a, b = (ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, label_smoothing=0.1, z_coef=1e-4) for _ in range(2))
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_token_out_of_range_is_reported(ctx):
    H, W, y, _ = _inputs(20, 64, 100)
    y[7] = 100
    ctx.rl_cross_entropy_fwd_bwd(H, W, y, None)
    s, detail = ctx.last_device_status()
    assert s == 7 and detail == 7
    assert ctx.last_device_status()[0] == 0


def test_dW_rows_are_reported(ctx):
    """The hook of the loss calls, for an fp32 dW; a bf16 one is refused with it."""
    from paper_2512_21450_b200 import RLHeadError
    H, W, y, mask = _inputs(200, 960, 900, seed=15)
    want = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask)["dW"]
    seen = []
    ctx.set_dw_slab_hook(lambda slab, a, b: seen.append((a, b)))
    try:
        got = ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask)["dW"]
        with pytest.raises(RLHeadError) as e:
            ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, dW_bf16=True)
        assert e.value.status == 1
        ctx.rl_cross_entropy_fwd_bwd(H, W, y, mask, want_dW=False)
    finally:
        ctx.set_dw_slab_hook(None)
    assert seen and seen[0][0] == 0 and seen[-1][1] == 900 and torch.equal(got, want)


def test_autograd(ctx):
    from paper_2512_21450_b200.autograd import fused_cross_entropy
    H, W, y, mask = _inputs(100, 256, 500, seed=16, masked=0.2)
    ref = cross_entropy(H, W, y, mask, 0.1, 1e-3)
    h, w = H.clone().requires_grad_(), W.clone().requires_grad_()
    loss, logp = fused_cross_entropy(h, w, y, mask, label_smoothing=0.1, z_coef=1e-3)
    (3 * loss).backward()
    want, bound = ref["loss"]
    assert_within(loss.detach(), want, bound, "loss")
    for x, k in ((h.grad, "dH"), (w.grad, "dW")):
        # twice rounded to bf16
        assert_within(x, 3 * ref[k][0], 3 * (ref[k][1] + 2.0 ** -8 * (ref[k][0].abs() + ref[k][1])), k)
    # a frozen head
    h2 = H.clone().requires_grad_()
    loss, _ = fused_cross_entropy(h2, W, y, mask, label_smoothing=0.1, z_coef=1e-3)
    loss.backward()
    assert_within(h2.grad, ref["dH"][0], ref["dH"][1] + 2.0 ** -8 * (ref["dH"][0].abs() + ref["dH"][1]), "dH")
    with torch.no_grad():
        loss, _ = fused_cross_entropy(H, W, y, mask, label_smoothing=0.1, z_coef=1e-3)
    assert_within(loss, want, bound, "loss")


def test_large_logits_and_one_column(ctx):
    """Logits in the hundreds; rows whose softmax is one everywhere it matters."""
    H, W, y, _ = _inputs(64, 128, 600, seed=17, std=2.0, sure=0.0)
    _check(ctx, H, W, y, None, z_coef=1e-5)
    out = ctx.rl_cross_entropy_fwd_bwd(H[:, :64].contiguous(), W[:1, :64].contiguous(), torch.zeros_like(y), None)
    assert np.abs(out["logp"].cpu().numpy()).max() <= 1e-5


def test_nan_row_that_counts_shows(ctx):
    H, W, y, _ = _inputs(40, 128, 300, seed=18)
    H[3, 5] = float("nan")
    out = ctx.rl_cross_entropy_fwd_bwd(H, W, y, None)
    assert bool(torch.isnan(out["loss"]).all()) and bool(torch.isnan(out["logp"][3])) and bool(torch.isnan(out["dH"][3]).all())
    keep = torch.arange(40, device=DEV) != 3
    assert bool(torch.isfinite(out["logp"][keep]).all())
