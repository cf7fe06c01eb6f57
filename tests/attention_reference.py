"""Plain 64-bit forms of the attention layer's operators (torch, on the operands' device), for the tests of the kernels, and how far a
kernel may be off them."""
import math

import torch

UBF, U32 = 2.0 ** -8, 2.0 ** -24          # half a unit in the last place, relative


def rotary(x, positions, frequencies, interleaved=False, amplitude=1.0, backward=False):
    x, n = x.double(), frequencies.numel()
    t = positions.double()[:, None, None] * frequencies.double()
    c, s = amplitude * t.cos(), amplitude * t.sin() * (-1 if backward else 1)
    at = torch.arange(n, device=x.device)
    a, b = (2 * at, 2 * at + 1) if interleaved else (at, at + n)
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def runs_of(query_start, key_start, query_rows, key_rows):
    """(first, last query, first, last key) of every sequence."""
    if query_start is None:
        return [(0, query_rows, 0, key_rows)]
    qs = [min(max(int(v), 0), query_rows) for v in query_start]
    ks = qs if key_start is None else [min(max(int(v), 0), key_rows) for v in key_start]
    return [(qs[i], qs[i + 1], ks[i], ks[i + 1]) for i in range(len(qs) - 1)]


def hidden(queries, keys, causal, window, device):
    """[queries][keys]: whether the key is not seen."""
    i, j = torch.arange(queries, device=device)[:, None] + keys - queries, torch.arange(keys, device=device)
    h = torch.zeros(queries, keys, dtype=torch.bool, device=device)
    if causal:
        h = j > i
        if window:
            h = h | (j <= i - window)
    return h


def attention(q, k, v, query_start=None, key_start=None, causal=True, window=0, scale=None):
    """(y, lse, bound of |error of y|, bound of |error of lse|); rows of no sequence: NaN.

    A kernel's logit has an fp32 rounding per product summed (towards zero: two half units) and one of its scaling; exponential,
    sum and quotient are a few more; the probability is rounded to bf16 once, the result once."""
    T, H, D = q.shape
    K = k.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    q, k, v = q.double(), k.double(), v.double()
    y = torch.full((T, H, D), math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full((T, H), math.nan, dtype=torch.float64, device=q.device)
    off, off_lse = torch.zeros_like(y), torch.zeros_like(lse)
    for q0, q1, k0, k1 in runs_of(query_start, key_start, T, k.shape[0]):
        if q1 <= q0:
            continue
        for h in range(H):
            a, b, c = q[q0:q1, h], k[k0:max(k0, k1), h // (H // K)], v[k0:max(k0, k1), h // (H // K)]
            hide = hidden(q1 - q0, b.shape[0], causal, window, q.device)
            s = (a @ b.t() * scale).masked_fill(hide, -math.inf)
            z = torch.logsumexp(s, 1) if b.shape[0] else torch.full((q1 - q0,), -math.inf, dtype=torch.float64, device=q.device)
            p = torch.exp(s - torch.where(z > -math.inf, z, torch.zeros_like(z))[:, None])
            lse[q0:q1, h], y[q0:q1, h] = z, p @ c
            most = (scale * (a.abs() @ b.abs().t()).masked_fill(hide, 0)).amax(1) if b.shape[0] else torch.zeros_like(z)
            e = 2 * U32 * (D + 4) * most + U32 * (16 + 2 * b.shape[0] / 16 + 8 * torch.where(z > -math.inf, z.abs(), torch.zeros_like(z)))
            off_lse[q0:q1, h] = e
            off[q0:q1, h] = (UBF + 3 * e[:, None]) * (1 + UBF) * (p @ c.abs()) + UBF * (1 + 2 * UBF) * y[q0:q1, h].abs() + 1e-30
    return y, lse, off, off_lse


def attention_backward(dy, q, k, v, y, lse, query_start=None, key_start=None, causal=True, window=0, scale=None, operand=UBF):
    """((dq, dk, dv), bounds of their errors) with y and lse as they are given; rows of no sequence: NaN.

    As above; delta and dy v are sums of dim products in fp32; p and ds are off by `operand` of themselves at most
    as operands (rounded to bf16 once)."""
    T, H, D = q.shape
    S, K = k.shape[:2]
    G = H // K
    scale = 1 / math.sqrt(D) if scale is None else scale
    dy, q, k, v, y, lse = (t.double() for t in (dy, q, k, v, y, lse))
    nan = lambda *s: torch.full(s, math.nan, dtype=torch.float64, device=q.device)  # noqa: E731
    out = [nan(T, H, D), nan(S, K, D), nan(S, K, D)]
    off = [torch.zeros_like(t) for t in out]
    for q0, q1, k0, k1 in runs_of(query_start, key_start, T, S):
        q1, k1 = max(q0, q1), max(k0, k1)
        if k1 > k0:
            out[1][k0:k1] = out[2][k0:k1] = 0
        if q1 > q0:
            out[0][q0:q1] = 0
        if q1 == q0 or k1 == k0:
            continue
        hide = hidden(q1 - q0, k1 - k0, causal, window, q.device)
        for h in range(H):
            a, g = q[q0:q1, h], dy[q0:q1, h]
            b, c = k[k0:k1, h // G], v[k0:k1, h // G]
            known = lse[q0:q1, h, None]
            known = torch.where(known > -math.inf, known, torch.zeros_like(known))
            p = torch.exp((a @ b.t() * scale).masked_fill(hide, -math.inf) - known)
            delta = (g * y[q0:q1, h]).sum(1, keepdim=True)
            ds = p * (g @ c.t() - delta)
            out[0][q0:q1, h] = scale * ds @ b
            out[1][k0:k1, h // G] += scale * ds.t() @ a
            out[2][k0:k1, h // G] += p.t() @ g
            e = 3 * (2 * U32 * (D + 4) * scale * (a.abs() @ b.abs().t()).masked_fill(hide, 0) + U32 * (16 + 4 * known.abs()))
            n = 2 * U32 * max(q1 - q0, k1 - k0) * G
            eds = (operand + e + n) * (1 + UBF) * ds.abs() + 2 * U32 * (D + 4) * p * (g.abs() @ c.t().abs() + (g * y[q0:q1, h]).abs().sum(1, keepdim=True))
            off[0][q0:q1, h] = scale * eds @ b.abs()
            off[1][k0:k1, h // G] += scale * eds.t() @ a.abs()
            off[2][k0:k1, h // G] += ((operand + e + n) * (1 + UBF) * p).t() @ g.abs()
    for o, t in zip(out, off):
        t += UBF * (1 + 2 * UBF) * torch.nan_to_num(o).abs() + 1e-30
    return out, off
