"""Workloads of the layer operators that make the per-node gradients: layer norm, 8-bit checkpoints, block-scaled products.

One node of data-parallel training holds a share of the step's tokens; K nodes are K runs of rows of one activation
matrix, and their gradients are K rows that the compression path reads.  The operators are

  norm        layer norm over the rows of x, its output also (or only) as an 8-bit matrix
  norm_grad   its backward pass: dx, and per node the gradients of the weight and the bias; x may be an 8-bit matrix
  checkpoint  x, optionally through a leaky ReLU, to an 8-bit matrix and back
  gate        a gradient times the derivative of the leaky ReLU whose 8-bit output is kept, in 16 and in 8 bits
  product     A B of two 8-bit matrices (B: the weights, read either way round), optionally through a leaky ReLU
  weight_grad per node dY^T X with X an 8-bit matrix

An 8-bit matrix holds e4m3 codes and, per block of 128 neighbours in a row (activations, gradients) or 128 x 128
entries (weights), a power of two 2^(s - 127) as the byte s: the smallest that brings the block's largest magnitude to
448 or less, 7 <= s <= 246; a block with an entry that is not finite has s = 255.

`own` chooses between the plain forms and the framework's kernels.  8-bit outputs come back as the float8 values that the bytes stand for.
"""
import math

import numpy as np
import torch
import torch.nn.functional as F

own = False

BLOCK = 128
SLOPE = 0.01      # of the leaky ReLU, the framework's activation
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token of a decode step, and a training batch that feeds an 8-bit product
        {"name": "norm_one_token", "op": "norm", "rows": 1, "cols": 4096, "type": "bf16", "y": True, "packed": True},
        {"name": "norm_batch", "op": "norm", "rows": 16384, "cols": 4096, "type": "bf16", "y": False, "packed": True},
        # an odd width in 32 bits over eight uneven nodes; a training batch whose input was kept in 8 bits
        {"name": "norm_grad_odd_nodes", "op": "norm_grad", "rows": 4099, "cols": 1001, "nodes": 8, "type": "fp32", "kept": False},
        {"name": "norm_grad_batch", "op": "norm_grad", "rows": 16384, "cols": 4096, "nodes": 8, "type": "bf16", "kept": True},
        # a small odd activation; the hidden layer of a training batch, and its gradient on the way back
        {"name": "checkpoint_odd", "op": "checkpoint", "rows": 301, "cols": 1537, "type": "fp32", "slope": SLOPE},
        {"name": "checkpoint_batch", "op": "checkpoint", "rows": 16384, "cols": 8192, "type": "bf16", "slope": 1.0},
        {"name": "gate_batch", "op": "gate", "rows": 16384, "cols": 8192, "type": "bf16"},
        # one token; a ragged batch in 32 bits; the wide layer forward with its activation, and its input gradient
        {"name": "product_one_token", "op": "product", "rows": 1, "inner": 4096, "cols": 4096, "across": False, "out": "bf16", "slope": 1.0},
        {"name": "product_odd_across", "op": "product", "rows": 777, "inner": 1160, "cols": 2043, "across": True, "out": "fp32", "slope": 1.0},
        {"name": "product_batch", "op": "product", "rows": 16384, "inner": 4096, "cols": 8192, "across": False, "out": "packed", "slope": SLOPE},
        # four uneven nodes of a small odd layer; a training batch of eight nodes
        {"name": "weight_grad_odd_nodes", "op": "weight_grad", "rows": 3001, "cols": 1000, "inner": 519, "nodes": 4},
        {"name": "weight_grad_batch", "op": "weight_grad", "rows": 16384, "cols": 4096, "inner": 4096, "nodes": 8},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, n if rng.random() < 0.5 else (n + 15) // 16 * 16))

    op = rng.choice(["norm", "norm_grad", "checkpoint", "gate", "product", "product", "weight_grad", "weight_grad"])
    kind = rng.choice(["bf16", "fp32"])
    rows = size(1, 16384)
    if op == "norm":
        y = rng.random() < 0.5
        return {"op": op, "rows": rows, "cols": size(64, 8192), "type": kind, "y": y, "packed": not y or rng.random() < 0.5}
    if op == "norm_grad":
        return {"op": op, "rows": rows, "cols": size(64, 8192), "nodes": rng.randint(1, 16), "type": kind, "kept": rng.random() < 0.5}
    if op == "checkpoint":
        return {"op": op, "rows": rows, "cols": size(64, 8192), "type": kind, "slope": rng.choice([1.0, SLOPE])}
    if op == "gate":
        return {"op": op, "rows": rows, "cols": size(64, 8192), "type": kind}
    if op == "product":
        return {"op": op, "rows": rows, "inner": size(64, 8192), "cols": size(64, 8192 if rows < 8192 else 4096),
                "across": rng.random() < 0.5, "out": rng.choice(["bf16", "fp32", "packed"]), "slope": rng.choice([1.0, SLOPE])}
    return {"op": op, "rows": rows, "cols": size(64, 4096), "inner": size(64, 4096), "nodes": rng.randint(1, 8)}


def work(case):
    T, C, op = case["rows"], case["cols"], case["op"]
    size = 4 if case.get("type") == "fp32" else 2
    packed = 1 + 1 / BLOCK                                    # bytes of an 8-bit entry with its share of the scale
    if op == "norm":
        out = (size if case["y"] else 0) + (packed if case["packed"] else 0)
        return {"bytes": T * C * (size + out) + 8 * T + 8 * C, "flops": 8 * T * C}
    if op == "norm_grad":
        return {"bytes": T * C * (2 * size + (packed if case["kept"] else size)) + 8 * T + 4 * C + 8 * case["nodes"] * C, "flops": 14 * T * C}
    if op == "checkpoint":
        return {"bytes": T * C * (2 * size + 2 * packed), "flops": 4 * T * C}
    if op == "gate":
        return {"bytes": T * C * (size + 1 + 2 + packed), "flops": 4 * T * C}
    I = case["inner"]
    if op == "product":
        out = {"bf16": 2, "fp32": 4, "packed": packed}[case["out"]]
        return {"bytes": T * I * packed + I * C + T * C * out, "flops": 2 * T * I * C}
    return {"bytes": 2 * T * C + T * I * packed + 4 * case["nodes"] * C * I, "flops": 2 * T * I * C}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(g, rows, cols):
    """A residual stream: unit noise, a few loud channels, an offset per row, now and then a row of zeros."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    loud = torch.rand(cols, generator=g, device="cuda") < 0.01
    x = torch.where(loud, 12 * x, x) + 0.2 * torch.randn(rows, 1, generator=g, device="cuda")
    return torch.where(torch.rand(rows, 1, generator=g, device="cuda") < 0.002, torch.zeros_like(x), x)


def _gradients(g, rows, cols):
    """Heavier tails than a Gaussian's, rows of different scale, rows of padding without any gradient."""
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.rand(rows, cols, generator=g, device="cuda").clamp_min(1e-3).log().abs()
    x = x * 1e-3 * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    return torch.where(torch.rand(rows, 1, generator=g, device="cuda") < 0.02, torch.zeros_like(x), x)


def _matrix(x, dtype):
    """`x` with its rows 16 bytes apart or a multiple of that, as a user allocates it."""
    each = 16 // torch.empty((), dtype=dtype).element_size()
    room = torch.zeros(x.shape[0], -(-x.shape[1] // each) * each, dtype=dtype, device=x.device)
    room[:, :x.shape[1]] = x.to(dtype)
    return room[:, :x.shape[1]]


def _packed_room(rows, cols, block_rows=1):
    """Codes and scales of an 8-bit matrix: rows 16 bytes apart or a multiple of that, scales a multiple of 4."""
    codes = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda")
    scales = torch.zeros(-(-rows // block_rows), -(-cols // (4 * BLOCK)) * 4, dtype=torch.uint8, device="cuda")
    return [codes, scales]


def _kept(x, block_rows=1):
    """An 8-bit matrix as an earlier call left it."""
    rows, cols = x.shape
    room = _packed_room(rows, cols, block_rows)
    codes, scales = _pack(x.float(), block_rows)
    room[0][:, :cols] = codes.view(torch.uint8)
    room[1][:, :scales.shape[1]] = scales.view(torch.uint8)
    return room


def _nodes(seed, rows, nodes):
    """Where each node's rows start: uneven shares, some of them empty."""
    r = np.random.RandomState(seed % (1 << 31))
    share = r.gamma(8.0, size=nodes) * (r.rand(nodes) > 0.05)
    at = np.floor(rows * np.concatenate([[0.0], np.cumsum(share)]) / max(share.sum(), 1e-9)).astype(np.int64)
    at[-1] = rows
    return np.minimum(at, rows)


def prepare(case, seed):
    g = _generator(seed)
    T, C, op = case["rows"], case["cols"], case["op"]
    dtype = TYPES.get(case.get("type"))
    st = {"case": dict(case)}
    if op in ("norm", "norm_grad"):
        x = _activations(g, T, C).to(dtype)
        st["gamma"] = 1 + 0.2 * torch.randn(C, generator=g, device="cuda")
        st["beta"] = 0.1 * torch.randn(C, generator=g, device="cuda")
        st["mean"], st["rstd"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    if op == "norm":
        st["x"] = _matrix(x, dtype)
        st["y"] = torch.empty_like(st["x"]) if case["y"] else None
        st["packed"] = _packed_room(T, C) if case["packed"] else None
    elif op == "norm_grad":
        var, mean = torch.var_mean(x.float(), dim=1, correction=0)
        st["mean"].copy_(mean)
        st["rstd"].copy_((var + EPS).rsqrt())
        st["dy"] = _matrix(_gradients(g, T, C), dtype)
        st["x"] = None if case["kept"] else _matrix(x, dtype)
        st["x8"] = _kept(x) if case["kept"] else None
        st["dx"] = torch.empty_like(st["dy"])
        at = _nodes(seed, T, case["nodes"])
        st["start"] = torch.from_numpy(at).cuda()
        # the weight and the bias lie side by side in a row of the nodes' gradients
        st["grads"] = torch.zeros(case["nodes"], 2 * C, device="cuda")
    elif op == "checkpoint":
        st["x"] = _matrix(_activations(g, T, C), dtype)
        st["packed"], st["y"] = _packed_room(T, C), torch.empty_like(st["x"])
    elif op == "gate":
        st["x"] = _matrix(_gradients(g, T, C), dtype)
        st["gate"] = _kept(F.leaky_relu(_activations(g, T, C), SLOPE))
        st["packed"], st["y"] = _packed_room(T, C), _matrix(torch.zeros(T, C, device="cuda"), torch.bfloat16)
    elif op == "product":
        I = case["inner"]
        weights = (2 * torch.rand(I if case["across"] else C, C if case["across"] else I, generator=g, device="cuda") - 1) / math.sqrt(I)
        st["a"] = _kept(_activations(g, T, I))
        st["b"] = _kept(weights, BLOCK)
        st["packed"] = _packed_room(T, C) if case["out"] == "packed" else None
        st["y"] = None if case["out"] == "packed" else _matrix(torch.zeros(T, C, device="cuda"), TYPES[case["out"]])
    else:
        I = case["inner"]
        st["dy"] = _matrix(_gradients(g, T, C), torch.bfloat16)
        st["x8"] = _kept(_activations(g, T, I))
        at = _nodes(seed, T, case["nodes"])
        st["start"], st["longest"] = torch.from_numpy(at).cuda(), int(np.diff(at).max())
        st["grads"] = torch.zeros(case["nodes"], C * I, device="cuda")
    return st


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _blocks(x, block_rows):
    """Rows x cols as (rows / block_rows, block_rows, cols / 128, 128), filled up with zeros."""
    rows, cols = x.shape
    x = F.pad(x, (0, -cols % BLOCK, 0, -rows % block_rows))
    return x.reshape(x.shape[0] // block_rows, block_rows, x.shape[1] // BLOCK, BLOCK)


def _pack(x, block_rows=1):
    """Codes (float8) and scales (float8, powers of two) of a matrix in 32 bits."""
    rows, cols = x.shape
    b = _blocks(x, block_rows)
    finite = torch.isfinite(b).all(3, keepdim=True).all(1, keepdim=True)
    most = b.abs().amax((1, 3), keepdim=True)
    most = torch.where(finite, most, torch.zeros_like(most))
    s = (((most.view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(7, 246)
    by = ((254 - s) << 23).view(torch.float32)
    codes = torch.where(finite, (b * by).clamp(-448, 448), torch.full_like(b, float("nan"))).to(torch.float8_e4m3fn)
    s = torch.where(finite, s, torch.full_like(s, 255)).to(torch.uint8)
    codes = codes.view(torch.uint8).reshape(b.shape[0] * block_rows, -1)[:rows, :cols].contiguous()
    return codes.view(torch.float8_e4m3fn), s[:, 0, :, 0].contiguous().view(torch.float8_e8m0fnu)


def _values(room, rows, cols, block_rows=1):
    """The 32-bit values of an 8-bit matrix."""
    codes = room[0][:rows, :cols].contiguous().view(torch.float8_e4m3fn).float()
    s = room[1][:, :-(-cols // BLOCK)].contiguous().view(torch.float8_e8m0fnu).float()
    b = _blocks(codes, block_rows) * s[:, None, :, None]
    return b.reshape(b.shape[0] * block_rows, -1)[:rows, :cols]


def _leaky(x, slope):
    return torch.where(x > 0, x, slope * x)


def _plain(st):
    c = st["case"]
    T, C, op = c["rows"], c["cols"], c["op"]
    if op == "norm":
        x = st["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = ((d * d).mean(1) + EPS).rsqrt()
        y = d * rstd[:, None] * st["gamma"] + st["beta"]
        out = {"mean": mean, "rstd": rstd}
        if c["y"]:
            out["y"] = y.to(st["x"].dtype)
        if c["packed"]:
            out["codes"], out["scales"] = _pack(y)
        return out
    if op == "norm_grad":
        x = _values(st["x8"], T, C) if c["kept"] else st["x"].float()
        dy = st["dy"].float()
        xhat = (x - st["mean"][:, None]) * st["rstd"][:, None]
        g = dy * st["gamma"]
        dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * st["rstd"][:, None]
        row, at = torch.arange(T, device=dy.device), st["start"]
        of = ((row >= at[:-1, None]) & (row < at[1:, None])).float()
        return {"dx": dx.to(st["dy"].dtype), "dgamma": of @ (dy * xhat), "dbeta": of @ dy}
    if op == "checkpoint":
        codes, scales = _pack(_leaky(st["x"].float(), c["slope"]))
        return {"y": _values([codes.view(torch.uint8), scales.view(torch.uint8)], T, C).to(st["x"].dtype)}
    if op == "gate":
        negative = st["gate"][0][:, :C] >= 128                       # the sign bit of the activation that was kept
        y = torch.where(negative, SLOPE * st["x"].float(), st["x"].float())
        codes, scales = _pack(y)
        return {"y": y.to(torch.bfloat16), "codes": codes, "scales": scales}
    if op == "product":
        I = c["inner"]
        a = _values(st["a"], T, I)
        b = _values(st["b"], I, C, BLOCK) if c["across"] else _values(st["b"], C, I, BLOCK).t()
        y = _leaky(a @ b, c["slope"])
        if c["out"] == "packed":
            codes, scales = _pack(y)
            return {"codes": codes, "scales": scales}
        return {"y": y.to(TYPES[c["out"]])}
    I, at = c["inner"], st["start"]
    dy, x = st["dy"].float(), _values(st["x8"], T, I)
    row = at[:-1, None] + torch.arange(st["longest"], device=dy.device)      # every node's rows, filled up to the longest
    of = (row < at[1:, None]).float()[:, :, None]
    row = row.clamp_max(T - 1)
    dw = (dy[row] * of).transpose(1, 2) @ x[row]
    return {"dw": dw.reshape(c["nodes"], C * I)}


# ---- the framework's operators -------------------------------------------------------------------------------------

def _float8(room, cols):
    """The bytes of an 8-bit matrix as the float8 values that they stand for (views)."""
    return room[0][:, :cols].view(torch.float8_e4m3fn), room[1][:, :-(-cols // BLOCK)].view(torch.float8_e8m0fnu)


def _framework(st):
    from paper_2103_08870_b200 import layers
    c = st["case"]
    T, C, op = c["rows"], c["cols"], c["op"]
    if op == "norm":
        packed = layers.Packed(*st["packed"], C) if c["packed"] else None
        layers.layer_norm(st["x"], st["gamma"], st["beta"], EPS, st["mean"], st["rstd"], y=st["y"], packed=packed)
        out = {"mean": st["mean"], "rstd": st["rstd"]}
        if c["y"]:
            out["y"] = st["y"]
        if c["packed"]:
            out["codes"], out["scales"] = _float8(st["packed"], C)
        return out
    if op == "norm_grad":
        x = layers.Packed(*st["x8"], C) if c["kept"] else st["x"]
        dgamma, dbeta = st["grads"][:, :C], st["grads"][:, C:]
        layers.layer_norm_backward(st["dy"], x, st["gamma"], st["mean"], st["rstd"], st["dx"], dgamma, dbeta, node_start=st["start"])
        return {"dx": st["dx"], "dgamma": dgamma, "dbeta": dbeta}
    if op == "checkpoint":
        packed = layers.Packed(*st["packed"], C)
        layers.pack(st["x"], packed, slope=c["slope"])
        layers.unpack(packed, st["y"])
        return {"y": st["y"]}
    if op == "gate":
        layers.pack(st["x"], layers.Packed(*st["packed"], C), slope=SLOPE, gate=layers.Packed(*st["gate"], C), y=st["y"])
        codes, scales = _float8(st["packed"], C)
        return {"y": st["y"], "codes": codes, "scales": scales}
    if op == "product":
        a = layers.Packed(*st["a"], c["inner"])
        b = layers.Packed(*st["b"], C if c["across"] else c["inner"], BLOCK)
        packed = layers.Packed(*st["packed"], C) if c["out"] == "packed" else None
        layers.product(a, b, y=st["y"], packed=packed, across=c["across"], slope=c["slope"])
        if packed is None:
            return {"y": st["y"]}
        codes, scales = _float8(st["packed"], C)
        return {"codes": codes, "scales": scales}
    layers.weight_gradient(st["dy"], layers.Packed(*st["x8"], c["inner"]), st["grads"], node_start=st["start"])
    return {"dw": st["grads"]}


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def _power(e):
    """2^e for whole numbers e, from the bits of a 64-bit number: library powers are not exact to the last bit."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(room, rows, cols, tall=1):
    code = room[0][:rows, :cols].to(torch.int64)
    e, m = (code >> 3) & 15, code & 7
    v = torch.where(e > 0, (8 + m).double() * _power(e - 10), m.double() * 2.0 ** -9)
    v = torch.where(code >= 128, -v, v)
    i = torch.arange(rows, device=v.device) // tall
    j = torch.arange(cols, device=v.device) // BLOCK
    return v * _power(room[1].to(torch.int64) - 127)[i][:, j]


def _exact_pack(y):
    """Codes and scales by their definition: nearest multiple of the code's last place, ties to even."""
    wide = torch.zeros(y.shape[0], -(-y.shape[1] // BLOCK) * BLOCK, dtype=torch.float64, device=y.device)
    wide[:, :y.shape[1]] = y
    most = wide.unflatten(1, (-1, BLOCK)).abs().amax(2)
    frac, e = torch.frexp(most / 448)                            # most / 448 = frac 2^e with 1/2 <= frac < 1
    e = torch.where(frac == 0.5, e - 1, e).clamp(-120, 119)
    e = torch.where(frac == 0, torch.full_like(e, -120), e)
    scale = _power(e)
    q = wide / scale.repeat_interleave(BLOCK, 1)
    last = _power(torch.frexp(q.abs().clamp_min(2.0 ** -6))[1] - 4)
    return (torch.round(q / last) * last)[:, :y.shape[1]], scale


def exact(case, seed):
    st = prepare(case, seed)
    T, C, op = case["rows"], case["cols"], case["op"]
    if op == "norm":
        x = st["x"].double()
        mean = x.sum(1) / C
        rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).sum(1) / C + EPS)
        y = (x - mean[:, None]) * rstd[:, None] * st["gamma"].double() + st["beta"].double()
        out = {"mean": mean, "rstd": rstd}
        if case["y"]:
            out["y"] = y
        if case["packed"]:
            out["codes"], out["scales"] = _exact_pack(y)
        return out
    if op == "norm_grad":
        x = _exact_values(st["x8"], T, C) if case["kept"] else st["x"].double()
        dy, rstd = st["dy"].double(), st["rstd"].double()[:, None]
        xhat = (x - st["mean"].double()[:, None]) * rstd
        g = dy * st["gamma"].double()
        dx = rstd * (g - g.sum(1, keepdim=True) / C - xhat * ((g * xhat).sum(1, keepdim=True) / C))
        at = st["start"].tolist()
        runs = [slice(lo, hi) for lo, hi in zip(at[:-1], at[1:])]
        return {"dx": dx, "dgamma": torch.stack([(dy * xhat)[r].sum(0) for r in runs]), "dbeta": torch.stack([dy[r].sum(0) for r in runs])}
    if op == "checkpoint":
        y = st["x"].double()
        q, scale = _exact_pack(torch.where(y > 0, y, y * np.float64(np.float32(case["slope"]))))
        return {"y": q * scale.repeat_interleave(BLOCK, 1)[:, :C]}
    if op == "gate":
        y = st["x"].double()
        y = torch.where(st["gate"][0][:, :C] >= 128, y * np.float64(np.float32(SLOPE)), y)
        codes, scales = _exact_pack(y)
        return {"y": y, "codes": codes, "scales": scales}
    I = case["inner"]
    if op == "product":
        a = _exact_values(st["a"], T, I)
        b = _exact_values(st["b"], I, C, BLOCK) if case["across"] else _exact_values(st["b"], C, I, BLOCK).t()
        y = torch.matmul(a, b)
        y = torch.where(y > 0, y, y * np.float64(np.float32(case["slope"])))
        if case["out"] == "packed":
            codes, scales = _exact_pack(y)
            return {"codes": codes, "scales": scales}
        return {"y": y}
    dy, x, at = st["dy"].double(), _exact_values(st["x8"], T, I), st["start"].tolist()
    return {"dw": torch.stack([torch.matmul(dy[lo:hi].t(), x[lo:hi]).reshape(-1) for lo, hi in zip(at[:-1], at[1:])])}
