"""Calls of one context from several streams and threads: its workspace and device block are one, so they follow one another."""
import threading
import time

import pytest
import torch

DEV = "cuda:0"


class _Torch:
    """What Context asks torch for, without a device: the current stream's handle, its id and whether it is captured."""

    def __init__(self, monkeypatch):
        self.handle, self.id, self.capturing, self.synchronised, self.device = 0, 0, False, 0, 0
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.device, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: self.handle, raising=False)
        monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: self.capturing, raising=False)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("Stream", (), dict(stream_id=self.id, cuda_stream=self.handle)))
        monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: setattr(self, "synchronised", self.synchronised + 1))

    def on(self, handle, id, capturing=False):
        self.handle, self.id, self.capturing = handle, id, capturing


class _Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name,) + args[1:])
            return 0
        return call


def _context():
    from paper_2512_21450_b200 import Context
    c = Context.__new__(Context)
    c.lib, c.handle, c._address, c._ws, c._stream, c.device = _Library(), None, 0, None, None, torch.device("cuda", 0)
    return c


def test_a_context_that_changes_streams_follows_the_one_it_leaves(monkeypatch):
    t, c = _Torch(monkeypatch), _context()
    c._bind_stream()                              # the first: nothing to follow
    t.on(0x5000, 35)                              # one of torch's streams
    c._bind_stream()
    c._bind_stream()                              # the same again
    t.on(0, 0)
    c._bind_stream()
    t.on(0x6000, 67, capturing=True)              # the library knows what is captured
    c._bind_stream()
    t.on(0, 0)
    c._bind_stream()
    assert c.lib.calls == [("rl_set_stream", 0), ("rl_follow_stream", 0x5000), ("rl_follow_stream", 0), ("rl_follow_stream", 0x6000),
                           ("rl_follow_stream", 0)] and t.synchronised == 0


def test_a_stream_of_somebody_else_may_be_gone_when_it_is_left(monkeypatch):
    t, c = _Torch(monkeypatch), _context()
    c._bind_stream()
    t.on(0x7000, 0x7000)                          # a stream that torch was handed: its id is its handle
    c._bind_stream()
    assert t.synchronised == 0
    t.on(0x5000, 35)
    c._bind_stream()
    assert t.synchronised == 1 and c.lib.calls[-1] == ("rl_set_stream", 0x5000)
    t.on(0, 0)
    c._bind_stream()
    assert t.synchronised == 1 and c.lib.calls[-1] == ("rl_follow_stream", 0)
    t.on(0x7000, 0x7000)
    c._bind_stream()
    t.on(0x6000, 67, capturing=True)              # no synchronisation while a graph is captured
    c._bind_stream()
    assert t.synchronised == 1 and c.lib.calls[-1] == ("rl_set_stream", 0x6000)


class _Workspace:
    def __init__(self, n):
        self.n, self.recorded = n, []

    def numel(self):
        return self.n

    def data_ptr(self):
        return 1 << 20

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


def test_every_stream_that_used_a_workspace_is_waited_for_before_its_memory_goes(monkeypatch):
    t, c = _Torch(monkeypatch), _context()
    monkeypatch.setattr(torch, "empty", lambda n, **kw: _Workspace(n))
    c._bind_stream()
    c._need_workspace(100)
    first = c._ws
    for handle, id in ((0x5000, 35), (0, 0), (0x6000, 67)):
        t.on(handle, id)
        c._bind_stream()
        c._need_workspace(100)
    assert c._ws is first and first.recorded == [0x5000, 0, 0x6000]
    c._need_workspace(200)
    assert c._ws is not first and t.synchronised == 0
    # one that torch does not own cannot be waited for later
    second = c._ws
    t.on(0x7000, 0x7000)
    c._bind_stream()
    c._need_workspace(200)
    assert t.synchronised == 0 and second.recorded == []
    c._need_workspace(300)
    assert t.synchronised == 1 and c._kept == ()
    # one that a graph writes to is kept, and nothing waits while the graph is captured
    t.on(0x5000, 35, capturing=True)
    c._bind_stream()
    third = c._ws
    c._need_workspace(400)
    assert c._kept == (third,) and t.synchronised == 1 and third.recorded == []


def test_a_capture_on_another_device_than_the_current_one_is_seen(monkeypatch):
    """A workspace that a graph of device 0 writes to is kept, whatever device is current at the call."""
    import contextlib
    t, c = _Torch(monkeypatch), _context()
    monkeypatch.setattr(torch, "empty", lambda n, **kw: _Workspace(n))
    captured = {0: False, 1: False}
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: captured[t.device])

    @contextlib.contextmanager
    def device(d):
        before, t.device = t.device, d.index
        yield
        t.device = before
    monkeypatch.setattr(torch.cuda, "device", device)
    c._bind_stream()
    c._need_workspace(100)
    first = c._ws
    t.device, captured[0] = 1, True
    c._bind_stream()
    c._need_workspace(200)
    assert c._kept == (first,) and t.device == 1
    captured[0], captured[1], second = False, True, c._ws     # and not what another device captures
    c._captured = False
    c._bind_stream()
    c._need_workspace(300)
    assert c._kept == (first,) and c._ws is not second


def _in_threads(work, n):
    raised = []

    def run(i):
        try:
            work(i)
        except BaseException as e:
            raised.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(n)]
    for x in threads:
        x.start()
    for x in threads:
        x.join(60)
    assert not raised and not any(x.is_alive() for x in threads), raised


def test_threads_take_turns_on_the_shared_context(monkeypatch):
    """A call of the module-level functions binds a stream, then a workspace, then launches, with the interpreter's lock given up in between."""
    import paper_2512_21450_b200 as rl
    from paper_2512_21450_b200 import autograd, binding

    made, inside, overlaps, seen = [], [], [], []

    class Shared:
        def __init__(self, device):
            time.sleep(0.05)
            made.append(device)
            self.turn = threading.RLock()

        def __getattr__(self, name):
            def call(*args, **kw):
                inside.append(name)
                time.sleep(0.002)
                if len(inside) > 1:
                    overlaps.append(list(inside))
                inside.remove(name)
                seen.append(name)
                z = torch.zeros(1)
                return dict(loss=z, dH=z, dW=z, logp=z.clone(), entropy=z.clone(), metrics=z.clone())
            return call
    monkeypatch.setattr(binding, "Context", Shared)
    monkeypatch.setattr(binding, "_default_ctx", {})
    x = torch.zeros(1)
    calls = [lambda: rl.rl_grpo_advantages(x, 1), lambda: rl.rl_token_logprobs(x, x, x),
             lambda: rl.rl_policy_loss_fwd_bwd(x, x, x, x, x, x, x, 0.2, 0.2, 0.0), lambda: rl.rl_cross_entropy_fwd_bwd(x, x, x),
             lambda: rl.rl_quantize_rows(x), lambda: rl.rl_int8_matmul(x, x, x, x), lambda: rl.rl_int8_linear(x, x, x),
             lambda: rl.rl_token_logprobs_int8(x, x, x, x), lambda: autograd.fused_cross_entropy(x, x, x),
             lambda: autograd.fused_grpo_head_loss(x, x, x, x, x, x, x)]
    _in_threads(lambda i: [calls[(i + k) % len(calls)]() for k in range(len(calls))], 6)
    assert made == [0] and not overlaps and len(seen) == 6 * len(calls)


def test_no_context_is_refused():
    from paper_2512_21450_b200 import build
    from paper_2512_21450_b200.binding import load_library
    build.build()
    assert load_library().rl_follow_stream(None, None) == 1


def _data(T, d, V, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    H = torch.randn(T, d, generator=g, device=DEV).bfloat16()
    W = (torch.randn(V, d, generator=g, device=DEV) * 0.05).bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    return H, W, y, (torch.rand(T, generator=g, device=DEV) < 0.8).to(torch.uint8)


@pytest.mark.gpu
def test_two_streams_through_the_module_level_functions():
    """Different sizes on two streams, nothing synchronised in between: every result is that of a call alone."""
    import paper_2512_21450_b200 as rl
    H1, W1, y1, m1 = _data(900, 1024, 20000, 1)
    H2, W2, y2, m2 = _data(300, 512, 9000, 2)
    Wq, ws = rl.rl_quantize_rows(W2)

    def loss():
        out = rl.rl_cross_entropy_fwd_bwd(H1, W1, y1, m1, label_smoothing=0.1, z_coef=1e-4, dW_bf16=True)
        return [out[k] for k in ("loss", "logp", "lse", "dH", "dW")]

    def score():
        return list(rl.rl_token_logprobs_int8(H2, Wq, ws, y2, m2)) + [rl.rl_int8_linear(H2[:n], Wq, ws) for n in (300, 40)]
    want = []
    for call in (loss, score):
        want.append(call())
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        got.append((0, loss()))
        with torch.cuda.stream(side):
            got.append((1, score()))
    torch.cuda.synchronize()
    for i, outs in got:
        for a, b in zip(outs, want[i]):
            assert torch.equal(a, b), i
    assert rl.default_context(0).last_device_status()[0] == 0


@pytest.mark.gpu
def test_threads_through_the_module_level_functions():
    """Several threads, a stream and sizes of its own each, on the context that they share."""
    import paper_2512_21450_b200 as rl
    from paper_2512_21450_b200.autograd import fused_cross_entropy
    data = [_data(*s, i) for i, s in enumerate([(300, 512, 9000), (40, 1024, 5000), (700, 256, 3000)])]

    def calls(H, W, y, m):
        Wq, ws = rl.rl_quantize_rows(W)
        out = rl.rl_cross_entropy_fwd_bwd(H, W, y, m, label_smoothing=0.1)
        h = H.clone().requires_grad_()
        fused_cross_entropy(h, W, y, m)[0].backward()
        return [out[k] for k in ("loss", "logp", "dH", "dW")] + list(rl.rl_token_logprobs_int8(H, Wq, ws, y, m)) + [rl.rl_int8_linear(H, Wq, ws), h.grad]
    want = [calls(*x) for x in data]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for turn in range(8):
                got = calls(*data[i])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    wrong.append((i, turn))
    _in_threads(work, 3)
    assert not wrong and rl.default_context(0).last_device_status()[0] == 0


@pytest.mark.gpu
def test_memory_of_a_replaced_workspace_is_not_handed_out_while_another_stream_uses_it():
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        H, W, y, m = _data(500, 512, 6000, 5)
        side, done = torch.cuda.Stream(), torch.cuda.Event()
        other = Context(0)                            # loads the kernels, which may wait for the device
        with torch.cuda.stream(side):
            for n in (100, 500):
                other.rl_cross_entropy_fwd_bwd(H[:n], W, y[:n], m[:n])
        other.close()
        want = c.rl_cross_entropy_fwd_bwd(H[:100], W, y[:100], m[:100])
        address, size = c._ws.data_ptr(), c._ws.numel()
        cached = [torch.empty(size, dtype=torch.uint8, device=DEV).fill_(0) for _ in range(4)]
        del cached
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(3_000_000_000)          # more than a second
            got = c.rl_cross_entropy_fwd_bwd(H[:100], W, y[:100], m[:100])
            assert c._ws.data_ptr() == address
            c.rl_cross_entropy_fwd_bwd(H, W, y, m)
            assert c._ws.numel() > size
            done.record()
        assert not done.query()
        others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(5)]
        assert address not in [x.data_ptr() for x in others]
        for x in others:
            x.fill_(0xff)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)
    finally:
        c.close()


@pytest.mark.gpu
def test_two_streams_of_one_capture():
    """A captured stream that forks: the graph has the calls of both branches in the order in which they were made."""
    from paper_2512_21450_b200 import Context
    c = Context(0)
    try:
        H, W, y, m = _data(400, 512, 6000, 3)
        Wq, ws = c.rl_quantize_rows(W)
        loss, dH, dW = torch.empty(1, device=DEV), torch.empty_like(H), torch.empty_like(W)
        C = torch.empty(400, 6000, dtype=torch.bfloat16, device=DEV)
        ce = lambda: c.rl_cross_entropy_fwd_bwd(H, W, y, m, loss=loss, dH=dH, dW=dW, dW_bf16=True)  # noqa: E731
        logits = lambda: c.rl_int8_linear(H, Wq, ws, out=C)  # noqa: E731
        ce(), logits()
        want = [x.clone() for x in (loss, dH, dW, C)]
        torch.cuda.synchronize()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            main = torch.cuda.current_stream()
            side.wait_stream(main)
            ce()
            with torch.cuda.stream(side):
                logits()
            ce()
            main.wait_stream(side)
        for _ in range(3):
            for x in (loss, dH, dW, C):
                x.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip((loss, dH, dW, C), want))
        assert c.last_device_status()[0] == 0
        # calls that run follow on, and so does a stream that torch did not make
        ce()
        assert torch.equal(dW, want[2])
    finally:
        c.close()


@pytest.mark.gpu
def test_streams_made_by_somebody_else():
    """Handles from the runtime, destroyed by their owner before the context is used on another stream."""
    import ctypes
    from paper_2512_21450_b200 import Context
    runtime = ctypes.CDLL("libcudart.so.12")
    c = Context(0)
    try:
        H, W, y, m = _data(400, 512, 6000, 4)
        want = c.rl_cross_entropy_fwd_bwd(H, W, y, m)
        torch.cuda.synchronize()
        for _ in range(2):
            handle = ctypes.c_void_p()
            assert runtime.cudaStreamCreateWithFlags(ctypes.byref(handle), 1) == 0
            with torch.cuda.stream(torch.cuda.ExternalStream(handle.value)):
                a = c.rl_cross_entropy_fwd_bwd(H, W, y, m)
            torch.cuda.synchronize()
            assert c._foreign and runtime.cudaStreamDestroy(handle) == 0
            b = c.rl_cross_entropy_fwd_bwd(H, W, y, m)
            assert not c._foreign
            assert all(torch.equal(a[k], want[k]) and torch.equal(b[k], want[k]) for k in want)
    finally:
        c.close()
