"""Layer operators without a GPU: the plain 64-bit forms that the kernels are tested against, and what the library
refuses on the host before it enqueues anything."""
import contextlib
import ctypes as C

import numpy as np
import pytest
import torch

import layers_reference as R
from paper_2103_08870_b200 import build as B
from paper_2103_08870_b200 import lgc

OK, INVALID, WORKSPACE, UNSUPPORTED = 0, 1, 3, 4


@pytest.fixture(scope="module")
def lib():
    B.build()
    return lgc.lib()


def test_reference_codes_are_float8():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(R.code_values(codes), want)
    x = np.concatenate([np.random.RandomState(0).randn(4000) * s for s in (1e-3, 0.02, 1, 100)] + [want[np.isfinite(want)], [0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10]])
    x = np.clip(x, -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(R.nearest_code(x), want)


@pytest.mark.parametrize("tall", [1, 128])
def test_reference_blocks(tall):
    x = np.random.RandomState(1).randn(200, 300)
    codes, scales = R.pack(x, tall)
    assert scales.shape == (200 if tall == 1 else 2, 3)
    i, j = R.block_index(200, 300, tall)
    s = scales.astype(np.float64)[i, j]
    assert (np.abs(x) <= 448 * 2.0 ** (s - 127)).all()
    err = np.abs(R.unpack(codes, scales, tall) - x)
    assert (err <= np.maximum(np.abs(x) / 16, 2.0 ** (s - 127 - 10)) * (1 + 1e-12)).all()


def test_reference_layer_norm_is_pytorchs():
    r = np.random.RandomState(2)
    x, dy, gamma, beta = (torch.from_numpy(r.randn(*s)).requires_grad_() for s in ((5, 33), (5, 33), (33,), (33,)))
    y, mean, rstd = R.layer_norm(x.detach().numpy(), gamma.detach().numpy(), beta.detach().numpy(), 1e-5)
    want = torch.nn.functional.layer_norm(x, (33,), gamma, beta, 1e-5)
    np.testing.assert_allclose(y, want.detach().numpy(), atol=1e-12)
    want.backward(dy.detach())
    dx, xh = R.layer_norm_backward(dy.detach().numpy(), x.detach().numpy(), gamma.detach().numpy(), mean, rstd)
    np.testing.assert_allclose(dx, x.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose((dy.detach().numpy() * xh).sum(0), gamma.grad.numpy(), atol=1e-12)


def packed(codes=256, ld=256, scales=256, ld_scales=4):
    return C.byref(lgc.lgc_packed(codes, ld, scales, ld_scales))


def test_refused_on_the_host(lib):
    """Made-up device addresses: a call that is refused never uses them."""
    P = 4096
    pack = lambda x=P, t=0, r=4, c=256, ld=256, br=1, gate=None, out=packed(), y=None, ldy=0: lib.lgc_pack(x, t, r, c, ld, br, 1.0, gate, out, y, ldy, None)  # noqa: E731
    assert pack(x=None) == INVALID and pack(t=2) == INVALID and pack(r=-1) == INVALID and pack(c=0) == INVALID and pack(ld=255) == INVALID
    assert pack(x=P + 2) == INVALID and pack(br=64) == INVALID and pack(out=None) == INVALID and pack(br=128, gate=packed()) == INVALID
    assert pack(out=packed(codes=264)) == INVALID and pack(out=packed(ld=250)) == INVALID and pack(out=packed(scales=258)) == INVALID
    assert pack(out=packed(ld_scales=2)) == INVALID and pack(y=P + 1, ldy=256) == INVALID and pack(y=P, ldy=100) == INVALID
    assert pack(r=1 << 31) == INVALID and pack(r=0) == OK
    assert pack(br=128, r=65536 * 128) == UNSUPPORTED
    assert b"block" in lib.lgc_last_error(None)
    assert lib.lgc_unpack(None, 4, 256, 1, P, 0, 256, None) == INVALID
    assert lib.lgc_unpack(packed(), 4, 256, 1, P, 7, 256, None) == INVALID
    norm = lambda c=256, y=P, g=P, eps=1e-5, mean=P: lib.lgc_layer_norm(P, 0, 4, c, c, g, P, eps, y, c, None, mean, P, None)  # noqa: E731
    assert norm(y=None) == INVALID and norm(g=None) == INVALID and norm(eps=-1.0) == INVALID and norm(mean=P + 1) == INVALID
    assert norm(c=16385) == UNSUPPORTED and norm(eps=float("nan")) == INVALID
    n = C.c_size_t()
    assert lib.lgc_layer_norm_backward_scratch(4, 256, 0, C.byref(n)) == INVALID
    assert lib.lgc_layer_norm_backward_scratch(4, 256, 2, C.byref(n)) == OK and n.value >= 2 * 256 * 4
    back = lambda size=n.value, start=P, K=2, stride=256, scratch=P, xt=0, xp=None: lib.lgc_layer_norm_backward(  # noqa: E731
        P, 0, 256, P, xt, 256, xp, 4, 256, P, P, P, start, K, P, 256, P, P, stride, scratch, size, None)
    assert back(size=n.value - 1) == WORKSPACE and back(start=None) == INVALID and back(K=0) == INVALID and back(stride=255) == INVALID
    assert back(scratch=None) == INVALID and back(xt=2) == INVALID and back(start=P + 4) == INVALID
    prod = lambda a=packed(), b=packed(), across=0, r=4, c=256, i=256, y=P, t=0: lib.lgc_product(a, b, across, r, c, i, 1.0, y, t, 256, None, None)  # noqa: E731
    assert prod(a=None) == INVALID and prod(b=None) == INVALID and prod(across=2) == INVALID and prod(i=0) == INVALID and prod(y=None) == INVALID
    assert prod(i=257) == INVALID and prod(t=9) == INVALID and prod(r=0) == OK
    grad = lambda dy=P, ld=256, x=packed(), r=4, c=256, i=256, start=None, K=1, dw=P, stride=0, scratch=P, size=1 << 40: lib.lgc_weight_gradient(dy, ld, x, r, c, i, start, K, dw, stride, scratch, size, None)  # noqa: E731
    assert grad(dy=P + 2) == INVALID and grad(ld=260) == INVALID and grad(x=None) == INVALID and grad(K=2) == INVALID
    assert lib.lgc_weight_gradient_scratch(4, 256, 0, 1, C.byref(n)) == INVALID and lib.lgc_weight_gradient_scratch(4, 256, 256, 1, None) == INVALID
    assert lib.lgc_weight_gradient_scratch(4, 256, 256, 1, C.byref(n)) == OK and n.value >= 4 * 256 * 2
    assert grad(size=n.value - 1) == WORKSPACE and grad(scratch=None) == INVALID and grad(scratch=P + 8) == INVALID
    assert grad(start=P, K=2, stride=65535) == INVALID and grad(dw=None) == INVALID and grad(c=1 << 30, ld=1 << 30, i=2048, x=packed(ld=2048, ld_scales=16)) == INVALID


def test_a_gate_needs_a_slope_whose_sign_tells_the_branch(lib):
    """With a slope below zero, or -0, the result of a negative entry has no sign bit: its derivative cannot be read off."""
    pack = lambda slope, gate, rows=4: lib.lgc_pack(4096, 0, rows, 256, 256, 1, slope, gate, packed(), None, 0, None)  # noqa: E731
    for slope in (-0.01, -0.0, -1.0, float("-inf"), float("nan")):
        assert pack(slope, packed()) == INVALID
        assert b"slope" in lib.lgc_last_error(None)
        assert pack(slope, None, 0) == OK
    assert pack(0.0, packed(), 0) == OK and pack(0.01, packed(), 0) == OK


def test_binding_refuses_host_tensors():
    from paper_2103_08870_b200 import layers
    with pytest.raises(ValueError):
        layers.Packed(torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8))


class Stub:
    """What the binding asks of a CUDA tensor; there is no memory behind it."""

    is_cuda = True

    def __init__(self, *shape, dtype=torch.float32, device=0, ptr=4096):
        self.shape, self.dtype, self.device_index, self.ptr = shape, dtype, device, ptr
        self.device = torch.device("cuda", device)

    def get_device(self):
        return self.device_index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def stride(self, axis=None):
        s = tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))
        return s if axis is None else s[axis]

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.ptr


def test_scratch_is_allocated_on_the_stream_that_uses_it(monkeypatch):
    """The allocator hands out a block whose last user may still be queued on the stream that the block is allocated on."""
    from paper_2103_08870_b200 import layers
    current, at = ["current"], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    class Block(Stub):
        def record_stream(self, stream):
            pass

    def empty(n, **kw):
        at.append(current[-1])
        return Block(n, dtype=torch.uint8)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", empty)
    assert layers._scratch(64, None, None, Stub(4, 8))[1] == 64
    assert layers._scratch(64, None, "side", Stub(4, 8))[1] == 64
    assert at == ["current", "side"]


class NothingLaunched:
    """Stands in for the library: sizes are answered, a launch is a failure of the test."""

    def __getattr__(self, name):
        def call(*a):
            assert name.endswith("_scratch"), f"{name} was called"
            a[-1]._obj.value = 64
            return OK
        return call


def test_operands_and_streams_of_another_device_are_refused(monkeypatch):
    from types import SimpleNamespace
    from paper_2103_08870_b200 import layers
    monkeypatch.setattr(lgc, "lib", lambda: NothingLaunched())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    bf, i64, u8 = torch.bfloat16, torch.int64, torch.uint8
    R_, Cc, N = 4, 256, 256 * 256
    f = lambda d=0: Stub(R_, Cc, device=d)                                        # noqa: E731
    b = lambda d=0: Stub(R_, Cc, dtype=bf, device=d)                              # noqa: E731
    v = lambda n, d=0: Stub(n, device=d)                                          # noqa: E731
    p = lambda d=0, tall=1, rows=R_: layers.Packed(Stub(rows, Cc, dtype=u8, device=d), Stub(-(-rows // tall), 4, dtype=u8, device=d), Cc, tall)  # noqa: E731
    w = lambda d=0: p(d, 128, 256)                                                # noqa: E731
    g = lambda d=0, n=Cc: Stub(2, n, device=d)                                    # noqa: E731
    start = lambda d=0: Stub(3, dtype=i64, device=d)                              # noqa: E731
    room = lambda d=0: Stub(64, dtype=u8, device=d)                               # noqa: E731
    calls = [      # every operand in turn on the other device; the last time all of them
        (layers.pack, [f, p], dict(gate=p, y=b)), (layers.unpack, [p, f], {}),
        (layers.layer_norm, [f, lambda d=0: v(Cc, d), lambda d=0: v(Cc, d), 1e-5, lambda d=0: v(R_, d), lambda d=0: v(R_, d)], dict(y=f, packed=p)),
        (layers.layer_norm_backward, [f, f, lambda d=0: v(Cc, d), lambda d=0: v(R_, d), lambda d=0: v(R_, d), f, g, g], dict(node_start=start, scratch=room)),
        (layers.layer_norm_backward, [b, p, lambda d=0: v(Cc, d), lambda d=0: v(R_, d), lambda d=0: v(R_, d), b, g, g], dict(node_start=start, scratch=room)),
        (layers.product, [p, w], dict(y=f, packed=p)),
        (layers.weight_gradient, [b, p, lambda d=0: g(d, N)], dict(node_start=start, scratch=room)),
    ]
    for call, args, named in calls:
        slots = [i for i, a in enumerate(args) if callable(a)] + list(named)
        for other in [[s] for s in slots] + [slots]:
            at = lambda s, a: a(1 if s in other else 0) if callable(a) else a     # noqa: E731
            with pytest.raises(ValueError):
                call(*[at(i, a) for i, a in enumerate(args)], **{k: at(k, a) for k, a in named.items()})
        with pytest.raises(AssertionError):                                       # all where they belong: the library is called
            call(*[a() if callable(a) else a for a in args], **{k: a() for k, a in named.items()})
        with pytest.raises(ValueError):
            call(*[a() if callable(a) else a for a in args], **{k: a() for k, a in named.items()}, stream=SimpleNamespace(device_index=1, cuda_stream=0))
    with pytest.raises(ValueError):
        layers.Packed(Stub(R_, Cc, dtype=u8), Stub(R_, 4, dtype=u8, device=1), Cc)


def test_the_block_makes_its_device_current(monkeypatch):
    from paper_2103_08870_b200 import block
    seen = []

    class Stop(Exception):
        pass

    def stop(*a, **kw):
        raise Stop

    monkeypatch.setattr(torch.cuda, "set_device", seen.append)
    monkeypatch.setattr(torch, "Generator", stop)
    with pytest.raises(Stop):
        block.ResidualBlock(4, 8, 8, 1, device=torch.device("cuda", 1))
    assert seen == [torch.device("cuda", 1)]
