"""Rows in 8 bits, their products and scoring under a head held in 8 bits, against their definitions: integers and scales exactly,
products to the roundings that the definition names."""
import pytest
import torch

from tests.head_reference import HALF_STEP, assert_within, quantize_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module")
def ctx():
    from paper_2512_21450_b200 import Context
    c = Context(0)
    yield c
    c.close()


def _rows(T, d, dtype, seed=0, std=1.0):
    g = torch.Generator(DEV).manual_seed(seed)
    return (torch.randn(T, d, generator=g, device=DEV) * std).to(dtype)


def _ok(ctx):
    s, detail = ctx.last_device_status()
    assert s == 0, (s, hex(detail))


# ------------------------------------------------------------------ quantised rows
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,d", [(1, 1), (3, 7), (5, 16), (9, 255), (64, 1000), (33, 2048), (17, 2056), (1000, 3584), (4, 70001), (3, 70000), (5, 4096), (2, 4104), (40, 896)])
def test_rows_exactly(ctx, dtype, T, d):
    x = _rows(T, d, dtype, seed=T + d)
    Q, s = ctx.rl_quantize_rows(x)
    q, scale = quantize_rows(x)
    assert torch.equal(Q.double(), q) and torch.equal(s, scale)
    assert Q.stride(0) % 16 == 0 or T == 1


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_and_signs(ctx, dtype):
    """Multiples of halves of a row whose largest is 127: products that lie exactly between two integers go to the even one."""
    x = torch.arange(-127, 127.5, 0.5, device=DEV)[None].to(dtype)
    Q, s = ctx.rl_quantize_rows(x)
    assert s.item() == 1.0 and torch.equal(Q.double(), torch.round(x.double()))
    q, _ = quantize_rows(x * 3)
    assert torch.equal(ctx.rl_quantize_rows(x * 3)[0].double(), q)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_zeros_and_what_is_not_finite(ctx, dtype):
    x = _rows(8, 100, dtype)
    x[0] = 0
    x[1, 17] = float("inf")
    x[2, 99] = float("nan")
    x[3, 0] = float("-inf")
    x[4] = 0
    x[4, 5] = -0.0
    x[5] = 2.0 ** -24                       # a subnormal fp16
    x[6] = torch.finfo(dtype).max
    Q, s = ctx.rl_quantize_rows(x)
    q, scale = quantize_rows(x)
    assert torch.equal(Q.double(), q) and torch.equal(s.nan_to_num(-1), scale.nan_to_num(-1))
    assert s[0] == 0 and s[4] == 0 and bool(torch.isnan(s[1:4]).all()) and bool((Q[:5] == 0).all())
    assert bool((Q[5] == 127).all()) and bool((Q[6] == 127).all())
    if dtype != torch.float16:
        tiny = torch.tensor([[2.0 ** -100, -2.0 ** -101], [2.0 ** -101, 0.0]], device=DEV).to(dtype)
        Q, s = ctx.rl_quantize_rows(tiny)
        assert Q.tolist() == [[127, -64], [0, 0]] and s[1] == 0 and s[0] > 0


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_with_strides_and_what_lies_around_them(ctx, dtype):
    wide = _rows(20, 130, dtype, seed=3)
    x = wide[:, 1:98]                       # rows that start anywhere
    Q = torch.full((20, 112), -99, dtype=torch.int8, device=DEV)
    s = torch.empty(20, device=DEV)
    ctx.rl_quantize_rows(x, Q=Q[:, :97], scale=s)
    q, scale = quantize_rows(x)
    assert torch.equal(Q[:, :97].double(), q) and torch.equal(s, scale) and bool((Q[:, 97:] == -99).all())
    assert ctx.rl_quantize_rows(x[:0])[0].shape == (0, 97)


# ------------------------------------------------------------------ products
def _product(A, a, B, b):
    """Exact sums, rounded to fp32, times a, times b (fp32), before the last rounding."""
    n = A.double() @ B.double().T          # below 2^53
    return n.float() * a[:, None] * b[None, :], n


def _int8(T, d, seed, lo=-128):
    g = torch.Generator(DEV).manual_seed(seed)
    ld = (d + 15) // 16 * 16
    x = torch.full((T, ld), 111, dtype=torch.int8, device=DEV)   # behind the rows: what must not count
    x[:, :d] = torch.randint(lo, 128, (T, d), generator=g, device=DEV, dtype=torch.int8)
    return x[:, :d], torch.rand(T, generator=g, device=DEV) + 0.5


PRODUCTS = [(1, 1, 1), (1, 64, 7), (2, 17, 33), (3, 2048, 1000), (4, 100, 515), (5, 33, 2), (8, 1000, 4099), (7, 8000, 300), (8, 8192, 77),
            (8, 8193, 65), (9, 64, 1), (9, 1, 300), (16, 129, 256), (128, 256, 1000), (129, 256, 1000), (200, 1000, 4099), (300, 2048, 513), (257, 127, 8),
            (12, 3584, 40000), (33, 100, 1000), (40, 2048, 515), (64, 1024, 20011), (65, 130, 149), (100, 1024, 1500), (128, 900, 148), (17, 12000, 700), (33, 2560, 900), (48, 3200, 151), (64, 2432, 333), (96, 1408, 700), (81, 1500, 515),
            (128, 1024, 4099), (128, 1025, 300), (97, 256, 40000)]


@pytest.mark.parametrize("T,d,V", PRODUCTS)
@pytest.mark.parametrize("out", TYPES)
def test_product_exactly(ctx, T, d, V, out):
    (A, a), (B, b) = _int8(T, d, T + d), _int8(V, d, V + d + 1)
    want, _ = _product(A, a, B, b)
    C = torch.full((T, V), float("nan"), dtype=out, device=DEV)
    got = ctx.rl_int8_matmul(A, a, B, b, out_dtype=out, out=C)
    _ok(ctx)
    assert torch.equal(got, want.to(out))


@pytest.mark.parametrize("T", [2, 40, 300])
@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("V,ld,at", [(500, 520, 0), (500, 512, 3), (257, 259, 1), (64, 64, 0)])
def test_product_into_a_part_of_a_matrix(ctx, T, out, V, ld, at):
    (A, a), (B, b) = _int8(T, 200, 1), _int8(V, 200, 2)
    big = torch.full((T + 1, ld + at), 5.0, dtype=out, device=DEV)
    C = big[:T, at:at + V]
    ctx.rl_int8_matmul(A, a, B, b, out_dtype=out, out=C)
    _ok(ctx)
    assert torch.equal(C, _product(A, a, B, b)[0].to(out))
    assert bool((big[T] == 5).all()) and bool((big[:, :at] == 5).all()) and bool((big[:, at + V:] == 5).all())


@pytest.mark.parametrize("T", [1, 8, 9, 130])
def test_largest_sums(ctx, T):
    """Every product the largest there is: sums up to 2^31 - 2^14."""
    d = (1 << 17) - 1
    A = torch.full((T, d + 1), -128, dtype=torch.int8, device=DEV)[:, :d]
    B = torch.full((20, d + 1), -128, dtype=torch.int8, device=DEV)[:, :d]
    B[3] = 127
    one = torch.ones(T, device=DEV)
    got = ctx.rl_int8_matmul(A, one, B, torch.ones(20, device=DEV), out_dtype=torch.float32)
    _ok(ctx)
    want = torch.full((T, 20), float(128 * 128 * d), device=DEV)
    want[:, 3] = float(-128 * 127 * d)
    assert torch.equal(got, want)


@pytest.mark.parametrize("x_dtype", TYPES)
@pytest.mark.parametrize("T,d,V", [(1, 2048, 1001), (6, 100, 300), (33, 1000, 4099), (300, 512, 777), (1, 8, 1), (2, 136, 149), (12, 1000, 515),
                                   (13, 3584, 20000), (16, 4104, 333), (16, 10000, 300), (3, 7, 50), (17, 640, 2000)])
def test_linear(ctx, x_dtype, T, d, V):
    X, W = _rows(T, d, x_dtype, seed=1), _rows(V, d, torch.bfloat16, seed=2, std=0.05)
    Wq, ws = ctx.rl_quantize_rows(W)
    got = ctx.rl_int8_linear(X, Wq, ws, out_dtype=torch.float32)
    _ok(ctx)
    q, s = quantize_rows(X)
    assert torch.equal(got, _product(q, s, Wq, ws)[0])
    # and near the product that it stands for: every q is half an integer off at most
    exact = X.double() @ W.double().T
    qa, qw = s.double()[:, None] / 2, ws.double()[None, :] / 2
    bound = qa * W.double().abs().sum(1)[None, :] + qw * X.double().abs().sum(1)[:, None] + qa * qw * d
    assert_within(got, exact, bound * 1.001, "logits")


def test_nan_and_zero_tokens(ctx):
    for T in (4, 20):
        X, W = _rows(T, 128, torch.bfloat16, seed=5), _rows(300, 128, torch.bfloat16, seed=6)
        X[1, 3] = float("inf")
        X[2] = 0
        Wq, ws = ctx.rl_quantize_rows(W)
        out = ctx.rl_int8_linear(X, Wq, ws)
        assert bool(torch.isnan(out[1]).all()) and bool((out[2] == 0).all()) and bool(torch.isfinite(out[0]).all())
    assert ctx.rl_int8_linear(X[:0], Wq, ws).shape == (0, 300)


def test_half_precision_overflows_to_infinity(ctx):
    A = torch.full((2, 64), 127, dtype=torch.int8, device=DEV)
    out = ctx.rl_int8_matmul(A, torch.ones(2, device=DEV), A, torch.ones(2, device=DEV), out_dtype=torch.float16)
    assert bool(torch.isinf(out).all())


def test_offsets_past_32_bits(ctx):
    """More than 2^31 logits, and a B of more than 2^31 bytes."""
    T, V, d = 16384, 151936, 16
    (A, a), (B, b) = _int8(T, d, 3), _int8(V, d, 4)
    C = torch.empty(T, V, dtype=torch.bfloat16, device=DEV)
    ctx.rl_int8_matmul(A, a, B, b, out=C)
    _ok(ctx)
    for t in (0, 14000, T - 1):
        assert torch.equal(C[t], _product(A[t:t + 1], a[t:t + 1], B, b)[0][0].bfloat16())
    odd = torch.empty(T * V + 8, dtype=torch.bfloat16, device=DEV)[1:1 + T * V].view(T, V)   # not through the TMA unit
    ctx.rl_int8_matmul(A, a, B, b, out=odd)
    assert torch.equal(odd, C)
    del C, odd
    V, ld = 200000, 16384
    big = torch.empty(V, ld, dtype=torch.int8, device=DEV)
    big[:, :64] = torch.randint(-128, 128, (V, 64), device=DEV, dtype=torch.int8)
    b = torch.rand(V, device=DEV)
    for T in (2, 20):
        A, a = _int8(T, 64, 5)
        got = ctx.rl_int8_matmul(A, a, big[:, :64], b, out_dtype=torch.float32)
        assert torch.equal(got, _product(A, a, big[:, :64], b)[0])


def test_streams_and_graphs(ctx):
    X, W = _rows(5, 512, torch.bfloat16, seed=7), _rows(1000, 512, torch.bfloat16, seed=8)
    Wq, ws = ctx.rl_quantize_rows(W)
    out = ctx.rl_int8_linear(X, Wq, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = ctx.rl_int8_linear(X, Wq, ws)
    side.synchronize()
    assert torch.equal(again, out)
    C = torch.empty_like(out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.rl_int8_linear(X, Wq, ws, out=C)
    X2 = _rows(5, 512, torch.bfloat16, seed=9)
    X.copy_(X2)
    graph.replay()
    torch.cuda.synchronize()
    got = C.clone()
    assert torch.equal(got, ctx.rl_int8_linear(X2, Wq, ws))


def test_graphs_outlive_their_workspace():
    """Two graphs of one context, captured at different sizes, the second with a workspace that took the first's place; replayed in turn,
    with other memory written in between."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        X, W = _rows(300, 512, torch.bfloat16, seed=7), _rows(1000, 512, torch.bfloat16, seed=8)
        tok = torch.randint(0, 1000, (300,), device=DEV, dtype=torch.int32)
        Wq, ws = c.rl_quantize_rows(W)
        C = torch.empty(5, 1000, dtype=torch.bfloat16, device=DEV)
        dW = torch.empty(1000, 512, device=DEV)
        small = lambda: c.rl_int8_linear(X[:5], Wq, ws, out=C)  # noqa: E731
        large = lambda: c.rl_cross_entropy_fwd_bwd(X, W, tok, dW=dW)  # noqa: E731
        want = small().clone()
        graphs, addresses = [], []
        for call in (small, large):
            call()
            addresses.append(c._ws.data_ptr())
            torch.cuda.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                call()
        want_dW = dW.clone()
        c.rl_cross_entropy_fwd_bwd(torch.cat([X] * 4), W, torch.cat([tok] * 4))
        assert [w.data_ptr() for w in c._kept] == addresses and c._ws.data_ptr() not in addresses
        others = [torch.full((n,), 3.0, device=DEV) for n in (64, 1 << 12, 1 << 16, 1 << 20, 1 << 22) for _ in range(3)]
        for _ in range(2):
            C.zero_(), dW.zero_()
            graphs[0].replay()
            graphs[1].replay()
            torch.cuda.synchronize()
            assert torch.equal(C, want) and torch.equal(dW, want_dW) and all(bool((x == 3).all()) for x in others)
    finally:
        c.close()


def test_two_contexts_at_once():
    """Contexts of two threads on two streams, their kernels side by side."""
    import threading
    from paper_2512_21450_b200 import Context
    X, W = _rows(600, 1024, torch.bfloat16, seed=7), _rows(9000, 1024, torch.bfloat16, seed=8, std=0.05)
    tok = torch.randint(0, 9000, (600,), device=DEV, dtype=torch.int32)
    torch.cuda.synchronize()
    made, wrong = {}, []

    def work(i):
        c = Context(0)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for turn in range(6):
                Wq, ws = c.rl_quantize_rows(W)
                got = [c.rl_int8_linear(X[:n], Wq, ws) for n in (1, 40, 600)] + list(c.rl_token_logprobs_int8(X, Wq, ws, tok))
                ce = c.rl_cross_entropy_fwd_bwd(X, W, tok, label_smoothing=0.1, dW_bf16=True)
                got += [ce["loss"], ce["dH"], ce["dW"]]
                stream.synchronize()
                if turn == 0:
                    made[i] = got
                elif not all(torch.equal(a, b) for a, b in zip(got, made[i])):
                    wrong.append((i, turn))
        if c.last_device_status()[0] != 0:
            wrong.append((i, "status"))
        c.close()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and len(made) == 2 and all(torch.equal(a, b) for a, b in zip(made[0], made[1]))


# ------------------------------------------------------------------ scoring
@pytest.mark.parametrize("T,d,V", [(1, 64, 1), (1, 64, 300), (77, 192, 1000), (128, 2048, 3000), (129, 1024, 777), (700, 2176, 1500), (2000, 256, 5000),
                                   (2, 128, 2), (16, 2048, 50000), (17, 3584, 3001), (40, 256, 151), (48, 1024, 20000), (64, 2048, 4099), (64, 64, 40000),
                                   (64, 2560, 3000), (33, 64, 17)])
def test_scoring(ctx, T, d, V):
    g = torch.Generator(DEV).manual_seed(T + d)
    W = _rows(V, d, torch.bfloat16, seed=1, std=0.05)
    tok = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    H = (_rows(T, d, torch.float32, seed=2) + 6 * torch.rand(T, 1, generator=g, device=DEV) / (0.0025 * d) * W[tok.long()].float()).bfloat16()
    mask = (torch.rand(T, generator=g, device=DEV) < 0.7).to(torch.uint8) if T > 1 else None
    if mask is not None:
        H[mask == 0] = float("nan")
        tok[mask == 0] = -5
    Wq, ws = ctx.rl_quantize_rows(W)
    logp, ent, lse = ctx.rl_token_logprobs_int8(H, Wq, ws, tok, mask)
    _ok(ctx)
    on = torch.ones(T, dtype=torch.bool, device=DEV) if mask is None else mask != 0
    q, s = quantize_rows(H[on])
    z = (q @ Wq.double().T) * s.double()[:, None] * ws.double()
    dz = 3 * HALF_STEP[torch.float32] * z.abs().amax(1)              # one rounding, two multiplications
    L = torch.logsumexp(z, 1)
    lp = z - L[:, None]
    dL = dz + 1e-6 * (L.abs() + 12)
    assert_within(lse[on], L, dL, "lse")
    assert_within(logp[on], lp.gather(1, tok[on].long()[:, None])[:, 0], dz + dL, "logp")
    p = lp.exp()
    E = -(p * lp).sum(1)
    # lse - sum p z, the sum with weights off by 2 (dz + 1e-6) at most
    assert_within(ent[on], E, dL + (p * z.abs()).sum(1) * 4 * (dz + 1e-6) + dz, "entropy")
    for x in (logp, ent, lse):
        assert bool((x[~on] == 0).all())


@pytest.mark.parametrize("T", [1, 20, 64, 100, 300])
def test_scoring_nothing_that_counts(ctx, T):
    """No valid row, or one, before and after calls that have more."""
    W = _rows(3000, 448, torch.bfloat16, seed=1, std=0.05)
    H = _rows(T, 448, torch.bfloat16, seed=2)
    tok = torch.randint(0, 3000, (T,), device=DEV, dtype=torch.int32)
    Wq, ws = ctx.rl_quantize_rows(W)
    want = [x.clone() for x in ctx.rl_token_logprobs_int8(H, Wq, ws, tok)]
    for _ in range(3):
        for x in ctx.rl_token_logprobs_int8(H, Wq, ws, tok, torch.zeros(T, dtype=torch.uint8, device=DEV)):
            assert bool((x == 0).all())
        one = torch.zeros(T, dtype=torch.uint8, device=DEV)
        one[T - 1] = 1
        for x, w in zip(ctx.rl_token_logprobs_int8(H, Wq, ws, tok, one), want):
            assert abs((x[T - 1] - w[T - 1]).item()) <= 4e-6 * (1 + abs(w[T - 1].item())) and bool((x[:T - 1] == 0).all())
        for x, w in zip(ctx.rl_token_logprobs_int8(H, Wq, ws, tok), want):
            assert torch.equal(x, w)
    assert ctx.rl_token_logprobs_int8(H[:0], Wq, ws, tok[:0])[0].shape == (0,)
    _ok(ctx)


@pytest.mark.parametrize("T", [5, 30, 77, 300])
def test_scoring_of_rows_that_are_not_finite(ctx, T):
    """Such a row's results are NaN, every other row's what they are without it."""
    W = _rows(2000, 256, torch.bfloat16, seed=1, std=0.05)
    H = _rows(T, 256, torch.bfloat16, seed=2)
    tok = torch.randint(0, 2000, (T,), device=DEV, dtype=torch.int32)
    Wq, ws = ctx.rl_quantize_rows(W)
    want = ctx.rl_token_logprobs_int8(H, Wq, ws, tok)
    bad = H.clone()
    bad[1, 9], bad[3, 0] = float("nan"), float("-inf")
    keep = torch.ones(T, dtype=torch.bool, device=DEV)
    keep[1] = keep[3] = False
    for x, w in zip(ctx.rl_token_logprobs_int8(bad, Wq, ws, tok), want):
        assert bool(torch.isnan(x[~keep]).all()) and torch.equal(x[keep], w[keep])
    zero = H.clone()
    zero[2] = 0                                       # logits of zero: the uniform distribution
    logp, ent, lse = ctx.rl_token_logprobs_int8(zero, Wq, ws, tok)
    log_v = torch.log(torch.tensor(2000.0)).item()
    assert max(abs(logp[2].item() + log_v), abs(ent[2].item() - log_v), abs(lse[2].item() - log_v)) <= 1e-5


def test_weights_written_just_before(ctx):
    """The weights are fetched ahead of the tokens, but not ahead of the launch that writes them."""
    base = [ctx.rl_quantize_rows(_rows(40000, 1024, torch.bfloat16, seed=s, std=0.05)) for s in (1, 2)]
    H = _rows(100, 1024, torch.bfloat16, seed=3)
    tok = torch.randint(0, 40000, (100,), device=DEV, dtype=torch.int32)
    Wq, ws = torch.empty_like(base[0][0]), torch.empty_like(base[0][1])
    calls = (lambda q, s: ctx.rl_int8_linear(H[:5], q, s), lambda q, s: ctx.rl_int8_linear(H, q, s),
             lambda q, s: ctx.rl_token_logprobs_int8(H, q, s, tok)[0])
    want = [[f(*b).clone() for b in base] for f in calls]
    for f, w in zip(calls, want):
        for i in (0, 1, 0, 1):
            Wq.copy_(base[i][0]), ws.copy_(base[i][1])
            assert torch.equal(f(Wq, ws), w[i])
    # and by one of the library's own launches
    X = [_rows(40000, 1024, torch.bfloat16, seed=s, std=0.05) for s in (1, 2)]
    for f, w in zip(calls, want):
        for i in (0, 1, 0, 1):
            ctx.rl_quantize_rows(X[i], Q=Wq, scale=ws)
            assert torch.equal(f(Wq, ws), w[i])


def test_scoring_agrees_with_the_logits(ctx):
    """The stages as they are used together: quantised head, logits of a prompt, scores of its tokens."""
    W = _rows(2000, 512, torch.bfloat16, seed=1, std=0.05)
    H = _rows(300, 512, torch.bfloat16, seed=2)
    tok = torch.randint(0, 2000, (300,), device=DEV, dtype=torch.int32)
    Wq, ws = ctx.rl_quantize_rows(W)
    z = ctx.rl_int8_linear(H, Wq, ws, out_dtype=torch.float32).double()
    logp, _, lse = ctx.rl_token_logprobs_int8(H, Wq, ws, tok)
    assert (lse - torch.logsumexp(z, 1)).abs().max().item() <= 1e-6 * 20
    assert (logp - torch.log_softmax(z, 1).gather(1, tok.long()[:, None])[:, 0]).abs().max().item() <= 1e-6 * 40
    few = torch.cat([ctx.rl_int8_linear(H[i:i + 5], Wq, ws, out_dtype=torch.float32) for i in range(0, 300, 5)])
    assert torch.equal(few.double(), z)       # one path or the other, the same numbers
    # scored states of a rollout stored in 8 bits, then a supervised step on them
    Q, s = ctx.rl_quantize_rows(H)
    out = ctx.rl_cross_entropy_fwd_bwd(Q, W, tok, H_scale=s)
    assert torch.equal(ctx.rl_int8_matmul(Q, s, Wq, ws, out_dtype=torch.float32).double(), z)
    assert (out["logp"] - logp).abs().mean().item() < 0.1 and _isfinite(out)


def _isfinite(out):
    return all(bool(torch.isfinite(v).all()) for v in out.values())


def test_native_and_general_host_paths_agree(ctx, monkeypatch):
    """The calls as the native host half makes them, which handles these, and as they are marshalled in Python."""
    from paper_2512_21450_b200 import binding
    X, W = _rows(70, 192, torch.bfloat16, seed=1), _rows(500, 192, torch.bfloat16, seed=2, std=0.1)
    tok = torch.randint(0, 500, (70,), device=DEV, dtype=torch.int32)
    mask = (torch.arange(70, device=DEV) % 5 != 0).to(torch.uint8)
    weight, count = torch.rand(70, device=DEV), torch.tensor([55], dtype=torch.int64, device=DEV)
    seen = []

    class Watched:
        def __getattr__(self, name):
            def call(*args):
                out = getattr(native, name)(*args)
                seen.append((name, out is not NotImplemented))
                return out
            return call

    def calls():
        Q, s = ctx.rl_quantize_rows(W)
        odd, so = ctx.rl_quantize_rows(X[:, :99].float())
        out = [Q, s, odd, so, ctx.rl_quantize_rows(X[:1].half())[0]]
        for n in (70, 1):
            out += [ctx.rl_int8_linear(X[:n], Q, s, out_dtype=t) for t in TYPES]
            out += ctx.rl_token_logprobs_int8(X[:n], Q, s, tok[:n], mask[:n])
        hq, hs = ctx.rl_quantize_rows(X)
        out += [ctx.rl_int8_matmul(hq[:n], hs[:n], Q, s, out_dtype=t) for n in (70, 1) for t in TYPES]
        for kw in (dict(), dict(mask=mask, label_smoothing=0.1, z_coef=1e-3, token_count=count), dict(token_weight=weight, want_dW=False),
                   dict(dW_bf16=True, want_dH=False), dict(dH_fp32=True), dict(want_dH=False, want_dW=False)):
            got = ctx.rl_cross_entropy_fwd_bwd(X, W, tok, **kw)
            out += [got[k] for k in sorted(got)]
            got = ctx.rl_cross_entropy_fwd_bwd(hq, W, tok, H_scale=hs, **kw)
            out += [got[k] for k in sorted(got)]
        return out
    calls()   # the workspace is there
    native = binding._host
    monkeypatch.setattr(binding, "_host", Watched())
    a = calls()
    assert len(seen) == 4 + 8 + 6 + 12 and all(ok for _, ok in seen), seen
    monkeypatch.setattr(binding, "_host", binding._NoHostCalls())
    b = calls()
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert x.dtype == y.dtype and x.shape == y.shape and x.stride() == y.stride() and torch.equal(x, y)


def test_what_the_native_half_leaves_to_the_general_path(ctx):
    from paper_2512_21450_b200 import RLHeadError
    X, W = _rows(10, 128, torch.bfloat16, seed=1), _rows(60, 128, torch.bfloat16, seed=2)
    Q, s = ctx.rl_quantize_rows(W)
    ctx.rl_int8_linear(X, Q, s)
    for call in (lambda: ctx.rl_int8_linear(X.cpu(), Q, s), lambda: ctx.rl_int8_linear(X, Q.cpu(), s), lambda: ctx.rl_int8_linear(X, Q, s[:59]),
                 lambda: ctx.rl_int8_linear(X[:, :64], Q, s), lambda: ctx.rl_int8_matmul(Q, s[:9], Q, s), lambda: ctx.rl_int8_matmul(Q[:, :64], s, Q, s),
                 lambda: ctx.rl_int8_matmul(X, s[:10], Q, s), lambda: ctx.rl_quantize_rows(X.T), lambda: ctx.rl_quantize_rows(X.cpu()),
                 lambda: ctx.rl_token_logprobs_int8(X, Q, s, torch.zeros(9, dtype=torch.int32, device=DEV)),
                 lambda: ctx.rl_cross_entropy_fwd_bwd(X, W, torch.zeros(9, dtype=torch.int32, device=DEV)),
                 lambda: ctx.rl_cross_entropy_fwd_bwd(X.cpu(), W, torch.zeros(10, dtype=torch.int32, device=DEV))):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(RLHeadError) as e:
        ctx.rl_cross_entropy_fwd_bwd(X, W, torch.zeros(10, dtype=torch.int32, device=DEV), label_smoothing=1.0)
    assert e.value.status == 1
    with pytest.raises(RLHeadError) as e:
        ctx.rl_int8_linear(X, torch.zeros(60, 144, dtype=torch.int8, device=DEV)[:, 8:136], s)      # rows that start on 8 bytes
    assert e.value.status == 3


@pytest.mark.parametrize("T", [3, 40, 70, 300])
def test_slices_of_a_head(ctx, T):
    """Rows of a head from any one on, as a rank of a head that is split by vocabulary holds them: their scales start anywhere."""
    X, W = _rows(T, 256, torch.bfloat16, seed=1), _rows(900, 256, torch.bfloat16, seed=2, std=0.1)
    Q, s = ctx.rl_quantize_rows(W)
    whole = ctx.rl_int8_linear(X, Q, s, out_dtype=torch.float32)
    tok = torch.randint(0, 300, (T,), device=DEV, dtype=torch.int32)
    for a, b in ((0, 900), (1, 302), (301, 900), (599, 900)):
        assert torch.equal(ctx.rl_int8_linear(X, Q[a:b], s[a:b], out_dtype=torch.float32), whole[:, a:b])
        lse = ctx.rl_token_logprobs_int8(X, Q[a:b], s[a:b], tok)[2]
        assert (lse - torch.logsumexp(whole[:, a:b].double(), 1)).abs().max().item() <= 1e-6 * (lse.abs().max().item() + 12)
