"""The layer operators on the GPU against plain 64-bit forms: layer norm and its backward pass, 8-bit matrices, products,
weight gradients per node; their edge cases and what the binding refuses."""
import zlib

import numpy as np
import pytest
import torch

import layers_reference as R
from paper_2103_08870_b200 import layers, lgc

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8          # half a unit in the last place, relative: significands of 24 and 8 bits


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda").to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


def rng(*key):
    return np.random.RandomState(zlib.crc32(repr(key).encode()))


def view(t, ld, offset=0):
    """`t` in rows `ld` elements apart whose first element lies `offset` elements into its allocation."""
    room = torch.full((t.shape[0] * ld + offset + 64,), 7.0, device="cuda").to(t.dtype)
    v = room[offset:offset + t.shape[0] * ld].view(t.shape[0], ld)[:, :t.shape[1]]
    v.copy_(t)
    return v


def packed_of(codes, scales, cols=None, block_rows=1):
    """An 8-bit matrix on the GPU; what pads its rows must not matter."""
    rows, n = codes.shape
    p = layers.packed_empty(rows, n, block_rows)
    p.codes.fill_(0x7f)
    p.scales.fill_(255)
    p.codes[:, :n] = torch.from_numpy(codes).cuda()
    p.scales[:, :scales.shape[1]] = torch.from_numpy(scales).cuda()
    return p


def random_packed(r, rows, cols, block_rows=1, lo=100, hi=140):
    x = r.randn(rows, cols) * np.exp(r.randn(rows, 1))
    x[r.rand(rows, cols) < 0.02] = 0
    codes, _ = R.pack(x, block_rows)
    scales = r.randint(lo, hi, size=(-(-rows // block_rows), -(-cols // 128))).astype(np.uint8)
    return codes, scales


def bytes_of(p):
    return p.codes[:, :p.cols].cpu().numpy(), p.scales[:, :-(-p.cols // 128)].cpu().numpy()


# ---- 8-bit matrices ---------------------------------------------------------------------------------------------------

def awkward(r, rows, cols):
    x = (r.randn(rows, cols) * np.exp2(r.randint(-12, 12, size=(rows, 1)))).astype(np.float32)
    x[r.rand(rows, cols) < 0.1] = 0
    x[r.rand(rows, cols) < 0.05] *= -0.0
    if rows > 3:
        x[1] = 0                                        # a row without anything
        x[2] = 1e-40 * np.sign(x[2])                    # subnormal numbers
        x[3, ::2] = 3.3e38                              # beyond the largest scale: cut at 448
        x[3, 1::2] = -3.3e38
    if rows > 5 and cols > 2:
        x[4, cols // 2] = np.inf
        x[5, 0], x[5, cols - 1] = np.nan, -np.inf
    return x


@pytest.mark.parametrize("tall", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (7, 129), (130, 127), (300, 1537), (257, 384)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_pack_and_unpack_are_exact(rows, cols, tall, kind):
    r = rng(rows, cols, tall)
    x = dev(awkward(r, rows, cols), kind)
    for ld, offset in [(-(-cols // 8) * 8, 0), (cols + 3, 1)]:      # whole 16-byte rows, and rows that start anywhere
        xv = view(x, ld, offset)
        p = layers.packed_empty(rows, cols, tall)
        p.codes.fill_(0x55)
        y = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
        layers.pack(xv, p, y=y)
        codes, scales = R.pack(host(x), tall)
        got_codes, got_scales = bytes_of(p)
        assert np.array_equal(got_scales, scales)
        assert np.array_equal(got_codes, codes)
        assert (p.codes[:, cols:] == 0x55).all()                    # the padding is not the call's
        assert torch.equal(y.view(torch.int16)[~torch.isnan(x)], x.bfloat16().view(torch.int16)[~torch.isnan(x)])
        want = R.unpack(codes, scales, tall)
        for out in (torch.float32, torch.bfloat16):
            y = view(torch.zeros(rows, cols, dtype=out, device="cuda"), ld, offset)
            layers.unpack(p, y)
            np.testing.assert_array_equal(host(y), want)


def test_every_code_and_scale_is_exact_in_bf16():
    codes = np.tile(np.array([c for c in range(256) if c & 0x7f != 0x7f], np.uint8), (240, 1))
    scales = np.repeat(np.arange(7, 247, dtype=np.uint8)[:, None], 2, 1)
    p = packed_of(codes, scales)
    for kind in (torch.float32, torch.bfloat16):
        y = torch.empty(codes.shape, dtype=kind, device="cuda")
        layers.unpack(p, y)
        np.testing.assert_array_equal(host(y), R.unpack(codes, scales))


@pytest.mark.parametrize("rows,cols", [(1, 130), (37, 1000)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_pack_with_the_activation_and_its_derivative(rows, cols, kind):
    r = rng("act", rows, cols)
    x, g = dev(r.randn(rows, cols), kind), dev(1e-3 * r.randn(rows, cols), kind)
    x[0, :3] = torch.tensor([0.0, -0.0, -1e-30])
    slope = 0.01
    a, d = layers.packed_empty(rows, cols), layers.packed_empty(rows, cols)
    layers.pack(x, a, slope=slope)
    xs = host(x)
    act = np.where(xs > 0, xs, (np.float32(slope) * xs.astype(np.float32)).astype(np.float64))
    codes, scales = R.pack(act)
    assert np.array_equal(bytes_of(a)[0], codes) and np.array_equal(bytes_of(a)[1], scales)
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    layers.pack(g, d, slope=slope, gate=a, y=y)
    gs = host(g)
    want = np.where(codes >= 128, (np.float32(slope) * gs.astype(np.float32)).astype(np.float64), gs)
    codes, scales = R.pack(want)
    assert np.array_equal(bytes_of(d)[0], codes) and np.array_equal(bytes_of(d)[1], scales)
    assert torch.equal(y, dev(want.astype(np.float32)).bfloat16())
    # the derivative is that of the differences, away from the corner
    far = np.abs(xs) > 1e-3
    step = 1e-6
    f = lambda v: np.where(v > 0, v, np.float64(np.float32(slope)) * v)     # noqa: E731
    slopes = (f(xs + step) - f(xs - step)) / (2 * step)
    np.testing.assert_allclose((want / gs)[far & (gs != 0)], slopes[far & (gs != 0)], rtol=1e-6)


# ---- layer norm -------------------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (1, 4096), (5, 127), (33, 1000), (9, 1024), (17, 2049), (3, 8192), (2, 16384), (700, 257), (611, 1000), (600, 2050),
              (1201, 4096), (607, 401), (600, 5003), (593, 8200)]


def norm_inputs(r, rows, cols, kind):
    x = r.randn(rows, cols) * np.exp(r.randn(rows, 1)) + 10 * r.randn(rows, 1)
    x[:, r.rand(cols) < 0.02] *= 30
    if rows > 2:
        x[2] = 0.5                                      # a constant row: the variance is zero
    return dev(x, kind), dev(1 + 0.3 * r.randn(cols)), dev(0.2 * r.randn(cols))


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("aligned", [True, False])
def test_layer_norm(rows, cols, kind, aligned):
    r = rng("norm", rows, cols)
    x, gamma, beta = norm_inputs(r, rows, cols, kind)
    ld, offset = (-(-cols // 8) * 8, 0) if aligned else (cols + 1, 3)
    xv, y = view(x, ld, offset), view(torch.zeros_like(x), ld, offset)
    p = layers.packed_empty(rows, cols)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    layers.layer_norm(xv, gamma, beta, 1e-5, mean, rstd, y=y, packed=p)
    xs, gs, bs = host(x), host(gamma), host(beta)
    want, m, rs = R.layer_norm(xs, gs, bs, 1e-5)
    # sums of 32 entries one after the other and a tree of ten levels: 42 roundings, and the division
    terms = 44
    dm = terms * U32 * np.abs(xs).mean(1)
    assert (np.abs(host(mean) - m) <= dm + 1e-30).all()
    drs = (terms + 4) * U32 + 0.5 * (dm * rs) ** 2       # (a mean that is off adds its square to the variance)
    assert (np.abs(host(rstd) - rs) <= drs * rs).all()
    xh = np.abs((xs - m[:, None]) * rs[:, None])
    bound = np.abs(gs) * ((dm * rs)[:, None] + xh * (drs[:, None] + 4 * U32)) + 2 * U32 * np.abs(want) + 1e-30
    assert (np.abs(host(y) - want) <= bound * 1.01 + (UBF * 1.01 * np.abs(want) if kind == torch.bfloat16 else 0)).all()
    # in 8 bits: those of a result in fp32, which the 32-bit output is
    if kind == torch.float32:
        codes, scales = R.pack(host(y))
        assert np.array_equal(bytes_of(p)[0], codes) and np.array_equal(bytes_of(p)[1], scales)
    else:
        val = R.unpack(*bytes_of(p))
        most = np.maximum.reduceat(np.abs(want), np.arange(0, cols, 128), axis=1).repeat(128, 1)[:, :cols]
        assert (np.abs(val - want) <= np.maximum(np.abs(want) / 16, most * 2.0 ** -16) + 2 * bound).all()
    q = layers.packed_empty(rows, cols)
    layers.layer_norm(xv, gamma, beta, 1e-5, mean, rstd, packed=q)          # the 8-bit form alone
    assert np.array_equal(bytes_of(q)[0], bytes_of(p)[0])


def test_layer_norm_keeps_a_bad_row_to_itself():
    x, gamma, beta = norm_inputs(rng("bad"), 6, 700, torch.float32)
    x[3, 5] = float("inf")
    x[4, 600] = float("nan")
    y, p = torch.empty_like(x), layers.packed_empty(6, 700)
    mean, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    layers.layer_norm(x, gamma, beta, 1e-5, mean, rstd, y=y, packed=p)
    bad = torch.isnan(y).all(1).cpu().tolist()
    assert bad == [False, False, False, True, True, False] and torch.isfinite(y[[0, 1, 2, 5]]).all()
    assert (bytes_of(p)[1] == 255).all(1).tolist() == bad


NODES = {1: [0, None], 3: [0, 1, 1, None], 5: [0, 0, 7, 8, 8, None]}      # None: the number of rows; empty nodes among them


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 512), (40, 127), (700, 257), (33, 2048), (12, 3001), (9, 8192), (8, 16384)])
@pytest.mark.parametrize("nodes", [1, 3, 5])
@pytest.mark.parametrize("kind,xkind", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, "kept"),
                                        (torch.float32, torch.bfloat16)])
def test_layer_norm_backward(rows, cols, nodes, kind, xkind):
    r = rng("grad", rows, cols, nodes)
    x, gamma, _ = norm_inputs(r, rows, cols, torch.float32)
    dy = dev(1e-2 * r.randn(rows, cols) * np.exp(r.randn(rows, 1)), kind)
    start = np.minimum([rows if s is None else s for s in NODES[nodes]], rows)
    _, m, rs = R.layer_norm(host(x), 1.0, 0.0, 1e-5)
    mean, rstd = dev(m), dev(rs)
    if xkind == "kept":
        arg = layers.packed_empty(rows, cols)
        layers.pack(x, arg)
        xs = R.unpack(*bytes_of(arg))
    else:
        x = x.to(xkind)
        arg, xs = view(x, cols + 5, 1), host(x)
    stride = 2 * cols + 9
    grads = torch.full((nodes, stride), 3.0, device="cuda")
    dg, db = grads[:, 1:1 + cols], grads[:, 1 + cols:1 + 2 * cols]
    dyv = view(dy, -(-cols // 8) * 8) if rows % 2 else view(dy, cols + 1, 1)
    dx = torch.empty_like(dyv)
    layers.layer_norm_backward(dyv, arg, gamma, mean, rstd, dx, dg, db, node_start=torch.from_numpy(start).cuda() if nodes > 1 else None)
    ds, gs, m, rs = host(dy), host(gamma), host(mean), host(rstd)
    want, xh = R.layer_norm_backward(ds, xs, gs, m, rs)
    g, ax = np.abs(ds * gs), np.abs(xh)
    # xh: two roundings, the first relative to x - mean; sums of 16 entries and a tree of ten levels, a division
    bound = rs[:, None] * U32 * (8 * g + 34 * g.mean(1, keepdims=True) + ax * 40 * (g * ax).mean(1, keepdims=True)) + 1e-30
    assert (np.abs(host(dx) - want) <= bound * 1.01 + (UBF * 1.01 * np.abs(want) if kind == torch.bfloat16 else 0)).all()
    for k in range(nodes):
        part = slice(start[k], start[k + 1])
        # at most 9 rows a chunk here, 45 chunks a slice, 16 slices, and three roundings of a term
        tol = 75 * U32
        t, a = (ds * xh)[part].sum(0), np.abs(ds * xh)[part].sum(0)
        assert (np.abs(host(dg)[k] - t) <= tol * a + 1e-30).all()
        t, a = ds[part].sum(0), np.abs(ds[part]).sum(0)
        assert (np.abs(host(db)[k] - t) <= tol * a + 1e-30).all()
    assert (grads[:, 0] == 3).all() and (grads[:, 1 + 2 * cols:] == 3).all()
    # again, in place, with scratch of the caller's: the same bits
    before = grads.clone()
    scratch = torch.empty(layers.layer_norm_backward_scratch(rows, cols, nodes), dtype=torch.uint8, device="cuda")
    layers.layer_norm_backward(dyv, arg, gamma, mean, rstd, dyv, dg, db, node_start=torch.from_numpy(start).cuda() if nodes > 1 else None, scratch=scratch)
    assert torch.equal(dyv, dx) and torch.equal(grads, before)


def test_layer_norm_gradient_agrees_with_differences():
    r = rng("differences")
    rows, cols = 3, 40
    x, gamma, beta = norm_inputs(r, rows, cols, torch.float32)
    x[2] += dev(r.randn(cols))
    dy = dev(r.randn(rows, cols))
    xs, gs, bs, ds = host(x), host(gamma), host(beta), host(dy)
    _, m, rs = R.layer_norm(xs, gs, bs, 1e-5)
    dx, grads = torch.empty_like(x), torch.empty(1, 2 * cols, device="cuda")
    layers.layer_norm_backward(dy, x, gamma, dev(m), dev(rs), dx, grads[:, :cols], grads[:, cols:])
    loss = lambda x, g, b: (R.layer_norm(x, g, b, 1e-5)[0] * ds).sum()      # noqa: E731
    step = 1e-5
    for i, j in [(0, 0), (1, 17), (2, 39), (0, 21)]:
        e = np.zeros_like(xs)
        e[i, j] = step
        want = (loss(xs + e, gs, bs) - loss(xs - e, gs, bs)) / (2 * step)
        assert abs(want - host(dx)[i, j]) <= 1e-4 * np.abs(host(dx)).max()
    for j in (0, 5, 39):
        e = np.zeros(cols)
        e[j] = step
        want = [(loss(xs, gs + e, bs) - loss(xs, gs - e, bs)) / (2 * step), (loss(xs, gs, bs + e) - loss(xs, gs, bs - e)) / (2 * step)]
        assert abs(want[0] - host(grads)[0, j]) <= 1e-4 * np.abs(host(grads)).max()
        assert abs(want[1] - host(grads)[0, cols + j]) <= 1e-4 * np.abs(host(grads)).max()


def chunk_rows(rows, cols, nodes):
    """Rows that one thread adds up one after the other in the backward pass (the launcher's rule)."""
    per_sm = 1 if cols > 4096 else 2 if cols > 2048 else 4 if cols > 1024 else 8 if cols > 512 else 16
    return max(4, -(-rows // max(148, per_sm * 148 - nodes)))


def backward_within_bounds(ds, xs, gs, m, rs, start, bf16, dx, dg, db):
    """Outputs of layer_norm_backward against the formula; all in 64 bits on the GPU."""
    rows, cols = ds.shape
    xh = (xs - m[:, None]) * rs[:, None]
    g, gx = ds * gs, ds * gs * xh
    want = rs[:, None] * (g - g.mean(1, keepdim=True) - xh * gx.mean(1, keepdim=True))
    # xh: two roundings, the first relative to x - mean; a row's sums: 16 entries a thread at most, five shuffles, 16 warps, the
    # product with 1 / cols (which is rounded itself)
    bound = rs[:, None] * U32 * (8 * g.abs() + 40 * g.abs().mean(1, keepdim=True) + 44 * xh.abs() * gx.abs().mean(1, keepdim=True)) + 1e-30
    assert ((dx - want).abs() <= bound * 1.01 + (UBF * 1.01 * want.abs() if bf16 else 0)).all()
    chunk = chunk_rows(rows, cols, len(start) - 1)
    for k, (lo, hi) in enumerate(zip(start[:-1], start[1:])):
        # a chunk's rows, a slice's chunks (eight slices), the slices, three roundings of a term
        tol = (chunk + -(-max(0, hi - lo) // (8 * chunk)) + 1 + 8 + 3) * U32
        t, a = (ds * xh)[lo:hi].sum(0), (ds * xh)[lo:hi].abs().sum(0)
        assert ((dg[k] - t).abs() <= tol * a + 1e-30).all()
        t, a = ds[lo:hi].sum(0), ds[lo:hi].abs().sum(0)
        assert ((db[k] - t).abs() <= tol * a + 1e-30).all()


# Chunks of more rows than the ring of shared-memory slots has slots (9 rows and 5 slots; 17 and 8; 16 and 8; 28 and 8; 21 and 3; ...),
# for every thread layout, rows whose last bytes fill no 16, and (contiguous) results whose rows start anywhere.
@pytest.mark.parametrize("rows,cols", [(1200, 4100), (40000, 33), (16384, 1001), (4099, 4096), (3000, 8192), (2500, 500), (16000, 2047), (2000, 2050)])
@pytest.mark.parametrize("kind,xkind", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, "kept"),
                                        (torch.float32, "kept"), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("contiguous", [False, True])
def test_layer_norm_backward_of_many_rows(rows, cols, kind, xkind, contiguous):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + cols)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")                                  # noqa: E731
    x = normal(rows, cols) * normal(rows, 1).exp() + 3 * normal(rows, 1)
    dy = view((1e-2 * normal(rows, cols) * normal(rows, 1).exp()).to(kind), -(-cols // 8) * 8)
    gamma = 1 + 0.3 * normal(cols)
    mean, rstd = x.mean(1), (x.var(1, correction=0) + 1e-5).rsqrt()
    if xkind == "kept":
        arg, xs = layers.packed_empty(rows, cols), torch.empty_like(x)
        layers.pack(x, arg)
        layers.unpack(arg, xs)
    else:
        arg = xs = view(x.to(xkind), -(-cols // 8) * 8)
    start = [0, rows // 3, rows // 3, rows // 3 + 5, rows]
    dx = torch.empty(rows, cols, dtype=kind, device="cuda") if contiguous else torch.empty_like(dy)
    grads = torch.full((4, 2 * cols + 3), 3.0, device="cuda")
    at = torch.tensor(start, device="cuda")
    layers.layer_norm_backward(dy, arg, gamma, mean, rstd, dx, grads[:, :cols], grads[:, cols:2 * cols], node_start=at)
    backward_within_bounds(dy.double(), xs.double(), gamma.double(), mean.double(), rstd.double(), start, kind == torch.bfloat16, dx.double(),
                           grads[:, :cols].double(), grads[:, cols:2 * cols].double())
    assert (grads[:, 2 * cols:] == 3).all()
    before = grads.clone()
    layers.layer_norm_backward(dy, arg, gamma, mean, rstd, dy, grads[:, :cols], grads[:, cols:2 * cols], node_start=at)      # in place
    assert torch.equal(dy, dx) and torch.equal(grads, before)
    layers.check()


@pytest.mark.parametrize("rows,cols", [(50, 127), (33, 2048), (700, 257), (20, 9001)])
@pytest.mark.parametrize("start", [[7, 20], [0, 5, 9], [30, 30, 30], [3, 3, 12, 12, 33]])
@pytest.mark.parametrize("aligned", [True, False])
def test_layer_norm_backward_of_rows_in_no_nodes_run(rows, cols, start, aligned):
    r = rng("no node", rows, cols, len(start))
    x, gamma, _ = norm_inputs(r, rows, cols, torch.float32)
    start = [min(s, rows) for s in start]
    K = len(start) - 1
    ld, offset = (-(-cols // 8) * 8, 0) if aligned else (cols + 1, 1)
    dy, xv = view(dev(r.randn(rows, cols)), ld, offset), view(x, ld, offset)
    mean, rstd = x.mean(1), (x.var(1, correction=0) + 1e-5).rsqrt()
    dx, grads = torch.full_like(dy, 7.0), torch.full((K, 2 * cols), 3.0, device="cuda")
    layers.layer_norm_backward(dy, xv, gamma, mean, rstd, dx, grads[:, :cols], grads[:, cols:], node_start=torch.tensor(start, device="cuda"))
    backward_within_bounds(dy.double(), x.double(), gamma.double(), mean.double(), rstd.double(), start, False, dx.double(),
                           grads[:, :cols].double(), grads[:, cols:].double())
    layers.check()


# ---- products -----------------------------------------------------------------------------------------------------------

PRODUCTS = [(1, 1, 1), (1, 4096, 512), (2, 130, 40), (7, 1000, 513), (128, 128, 128), (129, 129, 640), (300, 777, 1160), (33, 260, 2100),
            (513, 384, 96), (17, 64, 4224), (1500, 1900, 200), (2304, 1024, 1100), (1025, 2560, 130), (2600, 2700, 520), (3, 384, 8192), (4, 129, 8193), (1, 2043, 1160)]


@pytest.mark.parametrize("rows,cols,inner", PRODUCTS)
@pytest.mark.parametrize("across", [False, True])
def test_product(rows, cols, inner, across):
    r = rng("product", rows, cols, inner, across)
    a_bytes, b_bytes = random_packed(r, rows, inner), random_packed(r, *((inner, cols) if across else (cols, inner)), block_rows=128)
    a, b = packed_of(*a_bytes), packed_of(*b_bytes, block_rows=128)
    A, B = R.unpack(*a_bytes), R.unpack(*b_bytes, 128)
    B = B if across else B.T
    want, size = A @ B, np.abs(A) @ np.abs(B)
    # exact products; a rounding (of the accumulator's kind: at most two units in the last place) per 32 of the sum
    bound = (inner / 32 + 8) * 2.0 ** -22 * size
    y = torch.empty(rows, cols, device="cuda")
    layers.product(a, b, y=y, across=across)
    assert (np.abs(host(y) - want) <= bound).all()
    yb = view(torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda"), cols + 3, 1)
    layers.product(a, b, y=yb, across=across)
    assert torch.equal(yb, y.bfloat16())
    # with the activation, in both forms at once: the 8-bit one is that of the fp32 one
    p, z = layers.packed_empty(rows, cols), torch.empty(rows, cols, device="cuda")
    p.codes.fill_(0x55)
    layers.product(a, b, y=z, packed=p, across=across, slope=0.01)
    assert torch.equal(z, torch.where(y > 0, y, y * np.float32(0.01)))
    codes, scales = R.pack(host(z))
    assert np.array_equal(bytes_of(p)[0], codes) and np.array_equal(bytes_of(p)[1], scales)
    assert (p.codes[:, cols:] == 0x55).all()
    q = layers.packed_empty(rows, cols)
    layers.product(a, b, packed=q, across=across, slope=0.01)
    assert np.array_equal(bytes_of(q)[0], codes)
    layers.check()


def test_product_of_extreme_scales_and_of_blocks_that_are_not_numbers():
    r = rng("extreme")
    rows, cols, inner = 130, 140, 300
    (ac, _), (bc, _) = random_packed(r, rows, inner), random_packed(r, cols, inner, 128)
    asc = r.randint(7, 247, size=(rows, 3)).astype(np.uint8)
    bsc = np.full((2, 3), 127, np.uint8)
    asc[:, 1:] = asc[:, :1]
    asc[5, 1] = 255
    ac[5, 128:256] = 0x7f
    bsc[1, 2] = 255
    bc[128:, 256:] = 0xff
    y = torch.empty(rows, cols, device="cuda")
    layers.product(packed_of(ac, asc), packed_of(bc, bsc, block_rows=128), y=y)
    A, B = R.unpack(ac, asc), R.unpack(bc, bsc, 128)
    want = A @ B.T
    assert np.isnan(want[5]).all() and np.isnan(want[:, 128:]).all() and np.isfinite(np.delete(want[:, :128], 5, 0)).all()
    got = host(y)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    size = np.abs(np.nan_to_num(A)) @ np.abs(np.nan_to_num(B)).T
    fine = np.isfinite(want) & (size < 1e38) & (size > 1e-30)
    assert fine.mean() > 0.5 and (np.abs(got - want)[fine] <= (inner / 32 + 8) * 2.0 ** -22 * size[fine]).all()


@pytest.mark.parametrize("rows,cols,inner,nodes", [(1, 1, 1, 1), (1, 130, 70, 3), (64, 128, 128, 1), (65, 128, 129, 3), (300, 257, 513, 5), (2500, 40, 200, 3),
                                                   (1100, 300, 64, 5), (0, 30, 20, 3), (9000, 70, 300, 1), (6000, 513, 90, 3)])
@pytest.mark.parametrize("stride_extra", [0, 5])
def test_weight_gradient(rows, cols, inner, nodes, stride_extra):
    r = rng("weights", rows, cols, inner, nodes)
    codes, scales = random_packed(r, rows, inner)
    x = packed_of(codes, scales) if rows else layers.packed_empty(0, inner)
    dy = view(dev(1e-3 * r.randn(rows, cols), torch.bfloat16), -(-cols // 8) * 8)
    start = np.minimum([rows if s is None else s for s in NODES[nodes]], rows)
    n = cols * inner
    grads = torch.full((nodes, n + stride_extra), 3.0, device="cuda")
    scratch = torch.full((layers.weight_gradient_scratch(rows, cols, inner, nodes),), 0xff, dtype=torch.uint8, device="cuda")
    layers.weight_gradient(dy, x, grads[:, :n], node_start=torch.from_numpy(start).cuda() if nodes > 1 else None, scratch=scratch)
    X, D = R.unpack(codes, scales) if rows else np.zeros((0, inner)), host(dy)
    for k in range(nodes):
        part = slice(start[k], start[k + 1])
        want, size = D[part].T @ X[part], np.abs(D[part]).T @ np.abs(X[part])
        count = start[k + 1] - start[k]
        # exact products; an accumulator rounding per 16 rows up to 1024 of them, then one addition each
        bound = (min(count, 1024) / 16 + count / 1024 + 4) * 2.0 ** -22 * size
        assert (np.abs(host(grads)[k, :n].reshape(cols, inner) - want) <= bound).all()
    assert (grads[:, n:] == 3).all()
    layers.check()


def test_weight_gradient_reads_only_a_nodes_own_rows():
    r = rng("own rows")
    rows, cols, inner = 200, 130, 140
    codes, scales = random_packed(r, rows, inner)
    start = [0, 70, 70, 130, rows]
    dy = 1e-3 * r.randn(rows, cols)
    dy[70:130:7] = np.inf                                # node 2's rows are no numbers
    dy[75, ::2] = np.nan
    scales[101], codes[101] = 255, 0x7f
    d = view(dev(dy, torch.bfloat16), 136)
    grads = torch.empty(4, cols * inner, device="cuda")
    layers.weight_gradient(d, packed_of(codes, scales), grads, node_start=torch.tensor(start, device="cuda"))
    X, D, got = R.unpack(codes, scales), host(d), host(grads).reshape(4, cols, inner)
    assert np.isnan(got[2]).any()
    assert (got[1] == 0).all()
    for k in (0, 3):
        part = slice(start[k], start[k + 1])
        assert (np.abs(got[k] - D[part].T @ X[part]) <= 16 * 2.0 ** -22 * (np.abs(D[part]).T @ np.abs(X[part]))).all()


def test_weight_gradient_of_every_code_and_scale():
    """The codes become bf16 inside the kernel: one row a sum, so that the result is the product itself."""
    codes = np.tile(np.array([c for c in range(256) if c & 0x7f != 0x7f], np.uint8), (240, 1))
    scales = np.repeat(np.arange(7, 247, dtype=np.uint8)[:, None], 2, 1)
    dy = view(dev(np.ones((240, 1)), torch.bfloat16), 8)
    grads = torch.empty(240, codes.shape[1], device="cuda")
    layers.weight_gradient(dy, packed_of(codes, scales), grads, node_start=torch.arange(241, device="cuda"))
    want = R.unpack(codes, scales)
    big = np.abs(want) >= 2.0 ** -126                    # (the tensor cores may take subnormal numbers for zero)
    np.testing.assert_array_equal(host(grads)[big], want[big])
    assert (np.abs(host(grads) - want)[~big] <= np.abs(want)[~big]).all()


# ---- more tiles than CTAs --------------------------------------------------------------------------------------------------

def operands(rows, inner, cols, across, seed):
    """8-bit operands and their product in 64 bits, on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    a, b = layers.packed_empty(rows, inner), layers.packed_empty(*((inner, cols) if across else (cols, inner)), 128)
    for p in (a, b):
        layers.pack(torch.randn(p.rows, p.cols, generator=g, device="cuda") * torch.randn(p.rows, 1, generator=g, device="cuda").exp(), p)
    A, B = (torch.empty(p.rows, p.cols, device="cuda") for p in (a, b))
    layers.unpack(a, A)
    layers.unpack(b, B)
    A, B = A.double(), B.double() if across else B.double().t()
    return a, b, A @ B, A.abs() @ B.abs()


# (17, 20000) and (100, 40000): single CTAs, more than 148 tiles of 128 columns; (5000, 4200): pairs, 340 tiles for 74
@pytest.mark.parametrize("rows,cols,inner", [(17, 20000, 300), (100, 40000, 1200), (5000, 4200, 4200), (5000, 4200, 130), (1, 700, 8000)])
@pytest.mark.parametrize("across", [False, True])
def test_product_of_several_tiles_per_cta(rows, cols, inner, across):
    a, b, want, size = operands(rows, inner, cols, across, rows + inner)
    y, p = torch.empty(rows, cols, device="cuda"), layers.packed_empty(rows, cols)
    layers.product(a, b, y=y, packed=p, across=across)
    # exact products; less than a unit in the last place per step of 32 of the magnitudes' sum, of 1024 terms at most, then a
    # half per addition (and at most 64 additions where the fp32 pipes make the product of one row, 32 partial sums in a tree)
    bound = (min(inner, 1024) / 32 + 1 + inner / 2048 + 1 + (inner / 64 + 5 if rows == 1 else 0)) * 2.0 ** -23 * size
    assert ((y.double() - want).abs() <= bound).all()
    again = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    layers.product(a, b, y=again, across=across)
    assert torch.equal(again, y.bfloat16())
    q = layers.packed_empty(rows, cols)
    layers.pack(y, q)
    n = -(-cols // 128)
    assert torch.equal(p.codes[:, :cols], q.codes[:, :cols]) and torch.equal(p.scales[:, :n], q.scales[:, :n])
    layers.check()


# 180, 180 and 160 tiles of 256 x 256 for 74 pairs; runs that end inside a stage of 64 rows, on its edge, that are empty, and longer
# than the ring of six stages
@pytest.mark.parametrize("cols,inner,start", [(1100, 1300, [0, 1000, 1000, 1640, 1641, 4000, 4064]), (1288, 1300, [0, 640, 1333, 4000, 4096, 4100]),
                                              (2000, 2560, [17, 5000, 5101])])
def test_weight_gradient_of_several_tiles_per_pair(cols, inner, start):
    rows = start[-1] + 9                                  # (the last rows are no node's)
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    dy = view(torch.randn(rows, cols, generator=g, device="cuda").bfloat16(), -(-cols // 8) * 8)
    x, X = layers.packed_empty(rows, inner), torch.empty(rows, inner, device="cuda")
    layers.pack(torch.randn(rows, inner, generator=g, device="cuda"), x)
    layers.unpack(x, X)
    dy[start[-1]:] = float("nan")
    K, n = len(start) - 1, cols * inner
    grads = torch.full((K, n + 4), 3.0, device="cuda")
    layers.weight_gradient(dy, x, grads[:, :n], node_start=torch.tensor(start, device="cuda"))
    for k, (lo, hi) in enumerate(zip(start[:-1], start[1:])):
        D, Xk = dy[lo:hi].double(), X[lo:hi].double()
        want, size = D.t() @ Xk, D.abs().t() @ Xk.abs()
        # less than a unit in the last place per step of 16 rows, of 512 at most, then a half per addition
        bound = (min(hi - lo, 512) / 16 + 1 + (hi - lo) / 1024 + 1) * 2.0 ** -23 * size
        assert ((grads[k, :n].view(cols, inner).double() - want).abs() <= bound).all()
    assert (grads[:, n:] == 3).all()
    layers.check()


# ---- long sums ----------------------------------------------------------------------------------------------------------

# The tensor cores' additions round towards zero: a step (32 terms of the product, 16 of the weight gradient) loses less than a
# unit in the last place of the sum so far, 2^-23 of it.  Terms of one sign and one distribution: after step j of n the sum is
# j / n of the segment's, so a segment loses less than (n + 1) / 2 * 2^-23 of itself (and a tenth for the terms' scatter), in
# the mean half of that; every addition of a segment in fp32 registers, to nearest, 2^-24 of the sum.
def one_sign_bounds(steps, segments):
    lost = 1.1 * (steps + 1) / 2 * 2.0 ** -23
    return lost + segments * U32, lost / 2 + segments * U32


@pytest.mark.parametrize("rows,cols,inner", [(1, 384, 16384), (130, 200, 8192), (130, 200, 16384), (1300, 2000, 16384)])
@pytest.mark.parametrize("across", [False, True])
def test_product_of_long_sums_of_one_sign(rows, cols, inner, across):
    g = torch.Generator(device="cuda")
    g.manual_seed(inner + rows)
    a, b = layers.packed_empty(rows, inner), layers.packed_empty(*((inner, cols) if across else (cols, inner)), 128)
    layers.pack(torch.rand(rows, inner, generator=g, device="cuda"), a)
    layers.pack(torch.rand(b.rows, b.cols, generator=g, device="cuda"), b)
    A, B = (torch.empty(p.rows, p.cols, device="cuda") for p in (a, b))
    layers.unpack(a, A)
    layers.unpack(b, B)
    want = A.double() @ (B.double() if across else B.double().t())
    y = torch.empty(rows, cols, device="cuda")
    layers.product(a, b, y=y, across=across)
    lost = (want - y.double()) / want
    most, mean = one_sign_bounds(1024 // 32, inner / 1024)          # at most 1024 terms are added up in tensor memory
    assert lost.abs().max() <= most and lost.mean().abs() <= mean
    layers.check()


@pytest.mark.parametrize("rows,cols,inner", [(16384, 128, 264), (16384, 1032, 1032)])
def test_weight_gradient_of_long_sums_of_one_sign(rows, cols, inner):
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    dy, x = torch.rand(rows, cols, generator=g, device="cuda").bfloat16(), layers.packed_empty(rows, inner)
    layers.pack(torch.rand(rows, inner, generator=g, device="cuda"), x)
    X = torch.empty(rows, inner, device="cuda")
    layers.unpack(x, X)
    want = dy.double().t() @ X.double()
    dw = torch.empty(1, cols * inner, device="cuda")
    layers.weight_gradient(dy, x, dw)
    lost = (want - dw.view(cols, inner).double()) / want
    most, mean = one_sign_bounds(512 // 16, rows / 512)             # at most 512 rows are added up in tensor memory
    assert lost.abs().max() <= most and lost.mean().abs() <= mean
    layers.check()


# ---- streams, refusals ---------------------------------------------------------------------------------------------------

def test_calls_run_on_the_stream_they_are_given():
    r = rng("stream")
    side = torch.cuda.Stream()
    x = dev(r.randn(64, 256), torch.bfloat16)
    w = layers.packed_empty(256, 256, 128)
    h, grads = layers.packed_empty(64, 256), torch.zeros(1, 256 * 256, device="cuda")
    mean, rstd = torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    one, zero = torch.ones(256, device="cuda"), torch.zeros(256, device="cuda")
    wt = dev(r.randn(256, 256))
    y, dx = torch.empty(64, 256, dtype=torch.bfloat16, device="cuda"), torch.empty(64, 256, dtype=torch.bfloat16, device="cuda")
    dgb = torch.empty(1, 512, device="cuda")

    def all_of_it(stream):
        layers.pack(wt, w, stream=stream)
        layers.layer_norm(x, one, zero, 1e-5, mean, rstd, packed=h, stream=stream)
        layers.product(h, w, y=y, stream=stream)
        layers.weight_gradient(y, h, grads, stream=stream)
        layers.layer_norm_backward(y, x, one, mean, rstd, dx, dgb[:, :256], dgb[:, 256:], stream=stream)
        layers.unpack(h, x, stream=stream)

    before = x.clone()
    all_of_it(None)
    torch.cuda.synchronize()
    first = [t.clone() for t in (y, grads, dx, dgb, x)]
    x.copy_(before)
    torch.cuda.synchronize()
    all_of_it(side)
    side.synchronize()
    for a, b in zip(first, (y, grads, dx, dgb, x)):
        assert torch.equal(a, b)


def test_scratch_of_calls_on_two_streams_at_a_time():
    """Without a scratch of the caller's: two calls of one size, on streams that do not wait for each other."""
    r = rng("two streams")
    rows, cols, inner = 8192, 512, 1024
    side = torch.cuda.Stream()
    dy = [dev(r.randn(rows, cols), torch.bfloat16) for _ in range(2)]
    x = [layers.packed_empty(rows, inner) for _ in range(2)]
    for p in x:
        layers.pack(dev(r.randn(rows, inner)), p)
    h = [dev(r.randn(rows, cols)) for _ in range(2)]
    gamma, mean, rstd = torch.ones(cols, device="cuda"), torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")

    def run(i, stream=None):
        layers.weight_gradient(dy[i], x[i], dw[i], stream=stream)
        layers.layer_norm_backward(dy[i], h[i], gamma, mean, rstd, dx[i], dgb[i][:, :cols], dgb[i][:, cols:], stream=stream)

    def outputs():
        return ([torch.zeros(1, cols * inner, device="cuda") for _ in range(2)], [torch.zeros_like(d) for d in dy],
                [torch.zeros(1, 2 * cols, device="cuda") for _ in range(2)])

    dw, dx, dgb = want = outputs()
    for i in range(2):
        run(i)
        torch.cuda.synchronize()
    for _ in range(20):
        dw, dx, dgb = got = outputs()
        torch.cuda.synchronize()
        run(0)
        run(1, side)
        run(0)
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    layers.check()


def test_calls_in_a_cuda_graph_repeat_their_bits():
    r = rng("graph")
    rows, cols, K = 300, 520, 3
    x, dy = dev(r.randn(rows, cols), torch.bfloat16), dev(r.randn(rows, cols), torch.bfloat16)
    one = dev(r.randn(1, cols), torch.bfloat16)
    gamma, beta = torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")
    w, w8 = dev(r.randn(cols, cols)), layers.packed_empty(cols, cols, 128)
    h, d8, h1 = layers.packed_empty(rows, cols), layers.packed_empty(rows, cols), layers.packed_empty(1, cols)
    mean, rstd, m1, r1 = (torch.empty(n, device="cuda") for n in (rows, rows, 1, 1))
    y, dh, dx = (torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    y1 = torch.zeros(1, cols, device="cuda")
    grads = torch.zeros(K, cols * cols + 2 * cols, device="cuda")
    start = torch.tensor([0, 100, 100, rows], device="cuda")

    def step():
        layers.pack(w, w8)
        layers.layer_norm(x, gamma, beta, 1e-5, mean, rstd, packed=h)
        layers.product(h, w8, y=y)
        layers.layer_norm(one, gamma, beta, 1e-5, m1, r1, packed=h1)
        layers.product(h1, w8, y=y1)
        layers.pack(dy, d8)
        layers.product(d8, w8, y=dh, across=True)
        layers.weight_gradient(dy, h, grads[:, :cols * cols], node_start=start)
        layers.layer_norm_backward(dh, x, gamma, mean, rstd, dx, grads[:, cols * cols:-cols], grads[:, -cols:], node_start=start)

    out = (y, y1, dh, dx, grads, mean, rstd)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for new in (False, True, True):
        if new:
            x.copy_(dev(r.randn(rows, cols), torch.bfloat16))
            start[1:3] = 37
            step()
        want = [t.clone() for t in out]
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
    layers.check()


def test_no_rows():
    gamma = torch.ones(40, device="cuda")
    x, empty = torch.empty(0, 40, device="cuda"), torch.empty(0, device="cuda")
    p = layers.packed_empty(0, 40)
    layers.layer_norm(x, gamma, gamma, 1e-5, empty, empty, y=x)
    layers.pack(x, p)
    layers.unpack(p, x)
    grads = torch.full((2, 80), 3.0, device="cuda")
    layers.layer_norm_backward(x, x, gamma, empty, empty, x, grads[:, :40], grads[:, 40:], node_start=torch.zeros(3, dtype=torch.int64, device="cuda"))
    assert (grads == 0).all()
    layers.product(p, layers.packed_empty(70, 40, 128), y=torch.empty(0, 70, device="cuda"))


def test_refusals():
    f = torch.zeros(4, 256, device="cuda")
    v4, v256 = torch.zeros(4, device="cuda"), torch.zeros(256, device="cuda")
    p, w = layers.packed_empty(4, 256), layers.packed_empty(256, 256, 128)
    bad = [
        lambda: layers.pack(f.double(), p), lambda: layers.pack(f.cpu(), p), lambda: layers.pack(f.t(), p), lambda: layers.pack(f[:3], p),
        lambda: layers.pack(f, p, y=f), lambda: layers.unpack(p, f[:, :100]),
        lambda: layers.layer_norm(f, v4, v256, 1e-5, v4, v4, y=f), lambda: layers.layer_norm(f, v256, v256, 1e-5, v256, v4, y=f),
        lambda: layers.layer_norm(f, v256, v256, 1e-5, v4, v4, y=f.bfloat16()),
        lambda: layers.layer_norm_backward(f, f, v256, v4, v4, f.bfloat16(), f[:1], f[:1]),
        lambda: layers.layer_norm_backward(f, f, v256, v4, v4, f, f[:2], f[:2]),
        lambda: layers.layer_norm_backward(f, f, v256, v4, v4, f, f[:2], f[:1], node_start=torch.zeros(3, dtype=torch.int64, device="cuda")),
        lambda: layers.layer_norm_backward(f, f, v256, v4, v4, f, f[:2], f[:2], node_start=torch.zeros(3, dtype=torch.int32, device="cuda")),
        lambda: layers.product(p, p, y=f), lambda: layers.product(p, w, y=f[:, :200]), lambda: layers.product(p, layers.packed_empty(256, 200, 128), y=f),
        lambda: layers.weight_gradient(f, p, torch.zeros(1, 256 * 256, device="cuda")),
        lambda: layers.weight_gradient(f.bfloat16(), p, torch.zeros(1, 256, device="cuda")),
        lambda: layers.Packed(p.codes, p.scales[:2]), lambda: layers.Packed(p.codes, p.scales, 257), lambda: layers.Packed(p.codes, p.scales, 256, 64),
        lambda: layers.Packed(p.codes.float(), p.scales),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    one = torch.zeros(1, 20000, device="cuda")
    wide = one[0]
    calls = [   # what the library itself refuses
        (lambda: layers.layer_norm(f, v256, v256, -1.0, v4, v4, y=f), 1),
        (lambda: layers.layer_norm(f, v256, v256, 1e-5, v4, v4), 1),
        (lambda: layers.layer_norm(one, wide, wide, 1e-5, v4[:1], v4[:1], y=one), 4),
        (lambda: layers.product(p, w), 1),
        (lambda: layers.pack(torch.zeros(4, 200, device="cuda"), layers.Packed(torch.zeros(4, 200, dtype=torch.uint8, device="cuda"), p.scales, 200)), 1),
        (lambda: layers.weight_gradient(torch.zeros(4, 257, dtype=torch.bfloat16, device="cuda"), p, torch.zeros(1, 257 * 256, device="cuda")), 1),
        (lambda: layers.weight_gradient(f.bfloat16(), p, torch.zeros(1, 256 * 256, device="cuda"), scratch=torch.zeros(16, dtype=torch.uint8, device="cuda")), 3),
        (lambda: layers.layer_norm_backward(f, f, v256, v4, v4, f, torch.zeros(1, 256, device="cuda"), torch.zeros(1, 256, device="cuda"),
                                            scratch=torch.zeros(16, dtype=torch.uint8, device="cuda")), 3),
    ]
    for call, status in calls:
        with pytest.raises(lgc.LGCError) as e:
            call()
        assert e.value.status == status
    layers.check()
