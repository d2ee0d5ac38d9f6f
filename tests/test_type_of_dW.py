"""The buffer of dW is the caller's, fp32 or bf16: its type is named, or the call is refused before anything is written."""
import ctypes
from ctypes import byref, c_void_p

import pytest

INVALID, SHAPE = 1, 2
A = 1 << 20      # an address that is never read


@pytest.fixture(scope="module")
def lib():
    from paper_2512_21450_b200 import build
    from paper_2512_21450_b200.binding import load_library
    build.build()
    return load_library()


def _call(lib, opts, dH=A, dW=A):
    """SHAPE: the options were taken, and the width, which is looked at next, is no multiple of 64."""
    ctx = ctypes.cast(ctypes.create_string_buffer(8192), c_void_p)      # zeros in place of a context
    return lib.rl_cross_entropy_fwd_bwd(ctx, A, 128, A, 128, A, None, 4, 96, 50, A, dH, dW, byref(opts) if opts is not None else None)


def test_a_dW_of_no_named_type_is_refused(lib):
    from paper_2512_21450_b200.binding import rl_ce_opts
    end = rl_ce_opts.dW_dtype.offset + rl_ce_opts.dW_dtype.size
    assert _call(lib, None) == INVALID
    for size in (rl_ce_opts.token_weight.offset, rl_ce_opts.accumulate_dW.offset, rl_ce_opts.dH_dtype.offset, rl_ce_opts.dW_dtype.offset, end - 1):
        o = rl_ce_opts(size)
        o.dW_dtype = 1                                                  # behind the struct's end: not seen
        assert _call(lib, o) == INVALID, size
        assert _call(lib, o, dW=None) == SHAPE, size                # nothing to name
    assert _call(lib, None, dW=None) == SHAPE and _call(lib, None, dH=None, dW=None) == SHAPE
    for size in (end, ctypes.sizeof(rl_ce_opts)):
        for kind in (0, 1):
            o = rl_ce_opts(size)
            o.dW_dtype = kind
            assert _call(lib, o) == SHAPE, (size, kind)


def test_zero_is_bf16_in_every_struct(lib):
    """Shown by what only an fp32 dW takes."""
    from paper_2512_21450_b200.binding import rl_ce_opts
    for size in (rl_ce_opts.dW_dtype.offset + 4, ctypes.sizeof(rl_ce_opts)):
        o = rl_ce_opts(size)
        o.accumulate_dW = 1
        assert _call(lib, o) == INVALID
        o.dW_dtype = 1
        assert _call(lib, o) == SHAPE
