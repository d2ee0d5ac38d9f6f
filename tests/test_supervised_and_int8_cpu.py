"""What the supervised loss and the 8-bit calls refuse, before anything reaches a GPU: the library checks its arguments first, so a block
of zeros in place of a context does."""
import ctypes
from ctypes import byref, c_size_t, c_void_p

import pytest
import torch

OK, INVALID, SHAPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4
A = 1 << 20      # addresses that are never read


@pytest.fixture(scope="module")
def lib():
    from paper_2512_21450_b200 import build
    from paper_2512_21450_b200.binding import load_library
    build.build()
    return load_library()


@pytest.fixture()
def ctx():
    block = ctypes.create_string_buffer(8192)
    yield ctypes.cast(block, c_void_p)


def _ce(lib, ctx, opts=None, **kw):
    from paper_2512_21450_b200.binding import rl_ce_opts
    a = dict(H=A, ldH=128, W=A, ldW=128, y=A, mask=None, T=4, d=128, V=50, loss=A, dH=A, dW=A) | kw
    o = None
    if opts is not None:
        o = rl_ce_opts(ctypes.sizeof(rl_ce_opts))
        for k, v in opts.items():
            setattr(o, k, v)
    return lib.rl_cross_entropy_fwd_bwd(ctx, *a.values(), byref(o) if o is not None else None)


def test_cross_entropy_refusals(lib, ctx):
    nan, inf = float("nan"), float("inf")
    for opts in (dict(label_smoothing=-0.1), dict(label_smoothing=1.0), dict(label_smoothing=nan), dict(z_coef=-1e-6), dict(z_coef=inf),
                 dict(z_coef=nan), dict(dH_dtype=2), dict(dH_dtype=-1), dict(dW_dtype=2), dict(dW_dtype=0, accumulate_dW=1),
                 dict(struct_size=4), dict(struct_size=4096)):
        assert _ce(lib, ctx, opts) == INVALID, opts
    assert _ce(lib, None) == INVALID
    for kw in (dict(loss=None), dict(W=None), dict(H=None), dict(y=None), dict(T=-1), dict(d=0), dict(V=0)):
        assert _ce(lib, ctx, {}, **kw) == INVALID, kw
    for kw in (dict(d=96), dict(ldH=64), dict(ldW=64), dict(T=1 << 30), dict(V=1 << 30)):
        assert _ce(lib, ctx, {}, **kw) == SHAPE, kw
    for kw in (dict(ldH=132), dict(ldW=130), dict(H=A + 8), dict(W=A + 2), dict(dH=A + 4), dict(dW=A + 4)):
        assert _ce(lib, ctx, {}, **kw) == ALIGN, kw
    assert _ce(lib, ctx, dict(H_scale=A), ldH=136) == ALIGN


def test_rows_refusals(lib, ctx):
    def call(c=ctx, X=A, t=0, ldX=100, N=3, d=100, Q=A, ldQ=112, s=A):
        return lib.rl_quantize_rows(c, X, t, ldX, N, d, Q, ldQ, s)
    assert call(c=None) == INVALID
    for kw in (dict(X=None), dict(Q=None), dict(s=None), dict(t=3), dict(t=-1), dict(N=-1), dict(d=0)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(ldX=99), dict(ldQ=96), dict(N=1 << 31), dict(d=1 << 30, ldX=1 << 30, ldQ=1 << 30)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(X=A + 1), dict(t=1, X=A + 2), dict(Q=A + 8), dict(ldQ=120), dict(s=A + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(N=0, X=None, Q=None, s=None) == OK


def test_product_refusals(lib, ctx):
    def mm(c=ctx, X=A, ldA=112, a=A, B=A, ldB=112, b=A, T=3, d=100, V=50, C=A, t=0, ldC=50):
        return lib.rl_int8_matmul(c, X, ldA, a, B, ldB, b, T, d, V, C, t, ldC)

    def lin(c=ctx, X=A, xt=0, ldX=100, B=A, ldB=112, b=A, T=3, d=100, V=50, C=A, t=0, ldC=50):
        return lib.rl_int8_linear(c, X, xt, ldX, B, ldB, b, T, d, V, C, t, ldC)
    for call in (mm, lin):
        assert call(c=None) == INVALID
        for kw in (dict(B=None), dict(b=None), dict(C=None), dict(T=-1), dict(d=0), dict(V=0), dict(t=3), dict(t=-1)):
            assert call(**kw) == INVALID, kw
        for kw in (dict(ldB=96), dict(ldC=49), dict(T=1 << 30), dict(V=1 << 30, ldC=1 << 30), dict(d=1 << 17, ldB=1 << 17)):
            assert call(**kw) == SHAPE, kw
        for kw in (dict(B=A + 8), dict(ldB=120), dict(b=A + 2), dict(C=A + 1), dict(t=1, C=A + 2)):
            assert call(**kw) == ALIGN, kw
        assert call(T=0, C=None) == OK
    for kw in (dict(X=None), dict(a=None)):
        assert mm(**kw) == INVALID, kw
    assert mm(ldA=96) == SHAPE and mm(ldA=104) == ALIGN and mm(X=A + 8) == ALIGN and mm(a=A + 2) == ALIGN
    assert lin() == WORKSPACE
    assert lib.rl_set_workspace(ctx, A, 3 * 112) == OK and lin() == WORKSPACE     # room for the rows and not for their scales
    need = c_size_t()
    assert lib.rl_workspace_bytes_int8_linear(ctx, 3, 100, byref(need)) == OK and need.value >= 3 * 112 + 12
    assert lib.rl_set_workspace(ctx, A, need.value) == OK
    for kw in (dict(X=None), dict(xt=3)):
        assert lin(**kw) == INVALID, kw
    assert lin(ldX=99) == SHAPE and lin(X=A + 1) == ALIGN
    assert lib.rl_workspace_bytes_int8_linear(ctx, -1, 100, byref(need)) == INVALID


def test_scoring_refusals(lib, ctx):
    def call(c=ctx, H=A, ldH=128, W=A, ldW=128, s=A, y=A, mask=None, T=3, d=128, V=50, lp=A, e=None, lse=None):
        return lib.rl_token_logprobs_int8(c, H, ldH, W, ldW, s, y, mask, T, d, V, lp, e, lse)
    assert call(c=None) == INVALID
    for kw in (dict(H=None), dict(W=None), dict(s=None), dict(y=None), dict(lp=None), dict(T=-1), dict(d=0), dict(V=0)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(d=100), dict(ldH=64), dict(ldW=112), dict(d=1 << 17, ldH=1 << 17, ldW=1 << 17)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(ldW=136), dict(W=A + 8), dict(H=A + 8), dict(s=A + 2)):
        assert call(**kw) == ALIGN, kw
    assert call(T=0) == OK


def test_workspace_queries(lib, ctx):
    need = c_size_t()
    for bad in ((-1, 64, 10, 0), (1, 0, 10, 0), (1, 64, 0, 0), (1, 64, 10, 2), (1, 64, 10, -1)):
        assert lib.rl_workspace_bytes_ce(ctx, *bad, byref(need)) == INVALID
    assert lib.rl_workspace_bytes_ce(ctx, 1, 64, 10, 0, None) == INVALID


def test_binding_refuses_what_does_not_fit():
    """The checks of the Python calls, on tensors of the host with nothing behind them."""
    from paper_2512_21450_b200.binding import Context
    class Library:
        def __getattr__(self, name):
            def call(*args):
                raise RuntimeError(f"{name} was called")
            return call

    c = Context.__new__(Context)
    c.lib = Library()
    c._bind_stream = lambda: None
    c.device, c._ws, c.handle, c._address = torch.device("cpu"), None, 0, 0
    H, W, y = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(9, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    Q, s = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    Wq, ws = torch.zeros(9, 64, dtype=torch.int8), torch.zeros(9)
    for args, kw in (((H.float(), W, y), {}), ((H, W.float(), y), {}), ((H, W[:, :32], y), {}), ((H, W, y.long()), {}), ((H, W, y[:3]), {}),
                     ((Q, W, y), {}), ((H, W, y), dict(H_scale=s)), ((Q, W, y), dict(H_scale=s[:3])), ((Q, W, y), dict(H_scale=s.double())),
                     ((H, W, y, torch.zeros(3, dtype=torch.uint8)), {}), ((H, W, y, torch.zeros(4)), {}), ((H, W, y), dict(token_weight=s[:2])),
                     ((H, W, y), dict(token_count=torch.zeros(1))), ((H, W, y), dict(accumulate_dW=True)),
                     ((H, W, y), dict(dW=torch.zeros(9, 64, dtype=torch.bfloat16))), ((H, W, y), dict(dW=torch.zeros(8, 64))),
                     ((H, W, y), dict(dH=torch.zeros(4, 64))), ((H.T.contiguous().T, W, y), {}), ((H, W.T.contiguous().T, y), {}),
                     ((H.to("meta"), W, y), {}), ((H, W, y.to("meta")), {})):
        with pytest.raises(AssertionError):
            c.rl_cross_entropy_fwd_bwd(*args, **kw)
    for args, kw in (((Q, s, Wq[:, :32], ws), {}), ((H, s, Wq, ws), {}), ((Q, s[:3], Wq, ws), {}), ((Q, s, Wq.float(), ws), {}),
                     ((Q, s, Wq, ws[:8]), {}), ((Q, s, Wq, ws), dict(out=torch.zeros(4, 9))), ((Q, s, Wq, ws), dict(out=torch.zeros(4, 8).bfloat16())),
                     ((Q.T.contiguous().T, s, Wq, ws), {}), ((Q, s, Wq, ws.to("meta")), {})):
        with pytest.raises(AssertionError):
            c.rl_int8_matmul(*args, **kw)
    for args in ((H, Wq[:, :32], ws), (H, W, ws), (H, Wq, ws.double())):
        with pytest.raises(AssertionError):
            c.rl_int8_linear(*args)
        with pytest.raises(AssertionError):
            c.rl_token_logprobs_int8(args[0], args[1], args[2], y)
    with pytest.raises(AssertionError):
        c.rl_token_logprobs_int8(H.float(), Wq, ws, y)
    with pytest.raises(AssertionError):
        c.rl_quantize_rows(H, Q=Q[:3])
    with pytest.raises(AssertionError):
        c.rl_quantize_rows(H.T.contiguous().T)
