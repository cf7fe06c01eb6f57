"""Workloads of the attention layer's operators: rotary positions, attention over sequences, its backward pass.

The rows of one activation matrix are the tokens of several sequences (sequence s has rows start[s] .. start[s + 1] - 1, a run
may be empty), and q, k, v are views of a linear layer's result: [rows][heads][dim] with any distance between rows and heads.

  rotary          y = R x: pairs of a head's first 2 n entries turned by position * frequency[i], times an amplitude; the pairs
                  are neighbours (interleaved) or half of the rotary part apart; the rest of a head passes through.  The backward
                  pass is the same with the opposite angle
  attention       y = softmax(scale q k^T) v within every sequence, and lse, the logarithm of the softmax's denominator, per row
                  and head; heads / kv_heads heads of q share a head of k and v.  causal: the last query sees all keys of its
                  sequence, the one before it one less, and so on; window: of those only the last `window`.  A row that sees
                  no key has y = 0 and lse = -inf
  attention_grad  its backward pass from q, k, v, y, lse and dy: dq, dk, dv (the shared heads' gradients added up)

`own` chooses between the plain forms and the framework's kernels.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE = 10000.0


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one token far into a long context; a training batch's q and k heads together, frequencies scaled for a longer
        # context; the gradient of part of an odd head in 32 bits
        {"name": "rotary_one_token", "op": "rotary", "rows": 1, "heads": 40, "dim": 128, "pairs": 64, "interleaved": False, "type": "bf16",
         "far": 1 << 20, "scaled": 1.0, "backward": False},
        {"name": "rotary_batch", "op": "rotary", "rows": 16384, "heads": 40, "dim": 128, "pairs": 64, "interleaved": False, "type": "bf16",
         "far": 16384, "scaled": 8.0, "backward": False},
        {"name": "rotary_part_of_odd_head", "op": "rotary", "rows": 4099, "heads": 12, "dim": 80, "pairs": 20, "interleaved": True, "type": "fp32",
         "far": 4099, "scaled": 1.0, "backward": True},
        # one token after 8192 others; sixteen sequences, a few new tokens each, at very different lengths
        _attention("attention_one_token", "attention", 1, 8192, 1, 32, 8, 128),
        _attention("attention_few_tokens", "attention", 37, 50001, 16, 24, 8, 64),
        # small odd sequences; a training batch; a long document; windows; queries over another sequence's keys, all visible
        _attention("attention_odd_sequences", "attention", 1999, 1999, 23, 12, 4, 40),
        _attention("attention_batch", "attention", 8192, 8192, 8, 32, 8, 128),
        _attention("attention_long", "attention", 16384, 16384, 1, 16, 4, 128),
        _attention("attention_across", "attention", 1501, 4003, 5, 16, 16, 64, causal=False),
        # the gradients: small odd sequences with a window, the training batch, the long document
        _attention("attention_grad_odd_window", "attention_grad", 1999, 1999, 23, 12, 2, 72, window=100),
        _attention("attention_grad_batch", "attention_grad", 8192, 8192, 8, 32, 8, 128),
        _attention("attention_grad_long", "attention_grad", 16384, 16384, 1, 16, 4, 128),
    ]


def _attention(name, op, queries, keys, sequences, heads, kv_heads, dim, causal=True, window=0):
    return {"name": name, "op": op, "queries": queries, "keys": keys, "sequences": sequences, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "causal": causal, "window": window}


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, min(hi, n if rng.random() < 0.5 else (n + 15) // 16 * 16))

    op = rng.choice(["rotary", "attention", "attention", "attention_grad", "attention_grad"])
    if op == "rotary":
        dim = 8 * rng.randint(4, 16)
        pairs = dim // 2 if rng.random() < 0.6 else rng.randint(1, dim // 2)
        return {"op": op, "rows": size(1, 16384), "heads": rng.randint(1, 40), "dim": dim, "pairs": pairs, "interleaved": rng.random() < 0.5,
                "type": rng.choice(["bf16", "fp32"]), "far": size(1000, 1 << 22), "scaled": rng.choice([1.0, 4.0, 8.0]), "backward": rng.random() < 0.5}
    kv_heads, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
    dim = rng.choice([64, 128, 8 * rng.randint(4, 16)])
    keys = size(1, 16384)
    queries = keys if op == "attention_grad" or rng.random() < 0.5 else size(1, 16384)
    while kv_heads > 1 and kv_heads * group * queries * keys > 16 * 16384 * 16384:
        kv_heads //= 2
    causal = rng.random() < 0.75
    case = _attention(None, op, queries, keys, rng.randint(1, max(1, min(32, queries))), kv_heads * group, kv_heads, dim, causal,
                      size(16, 4096) if causal and rng.random() < 0.3 else 0)
    del case["name"]
    return case


def _starts(rows, sequences, salt):
    """Where each sequence's rows start: uneven lengths, now and then an empty one."""
    r = np.random.RandomState((rows * 64 + sequences) * 2 + salt)
    share = r.gamma(2.0, size=sequences) * (r.rand(sequences) > 0.05)
    at = np.floor(rows * np.concatenate([[0.0], np.cumsum(share)]) / max(share.sum(), 1e-9)).astype(np.int64)
    at[-1] = rows
    return np.minimum(at, rows)


def _runs(case):
    """Starts of the sequences' queries and keys."""
    at = _starts(case["queries"], case["sequences"], 0)
    if case["queries"] == case["keys"]:
        return at, at
    return at, _starts(case["keys"], case["sequences"], 1)


def _pairs_seen(case):
    """Pairs of a query and a key that it sees."""
    n = 0
    for lq, lk in zip(*(np.diff(at) for at in _runs(case))):
        if not case["causal"]:
            n += int(lq) * int(lk)
            continue
        seen = np.maximum(np.arange(lq, dtype=np.int64) + 1 + lk - lq, 0)
        n += int((np.minimum(seen, case["window"]) if case["window"] else seen).sum())
    return n


def work(case):
    if case["op"] == "rotary":
        size = 4 if case["type"] == "fp32" else 2
        n = case["rows"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * size + 8 * case["rows"] + 8 * case["pairs"], "flops": 6 * case["rows"] * case["heads"] * case["pairs"]}
    D, H, K = case["dim"], case["heads"], case["kv_heads"]
    q, k = 2 * case["queries"] * H * D, 2 * case["keys"] * K * D
    lse, starts = 4 * case["queries"] * H, 16 * (case["sequences"] + 1)
    if case["op"] == "attention":
        return {"bytes": 2 * q + 2 * k + lse + starts, "flops": 4 * D * H * _pairs_seen(case)}
    return {"bytes": 4 * q + 4 * k + lse + starts, "flops": 10 * D * H * _pairs_seen(case)}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _gradients(g, rows, heads, dim):
    """Heavier tails than a Gaussian's, rows of different scale, rows of padding without any gradient."""
    x = torch.randn(rows, heads, dim, generator=g, device="cuda") * torch.rand(rows, heads, dim, generator=g, device="cuda").clamp_min(1e-3).log().abs()
    x = x * 1e-3 * torch.exp(0.5 * torch.randn(rows, 1, 1, generator=g, device="cuda"))
    return torch.where(torch.rand(rows, 1, 1, generator=g, device="cuda") < 0.02, torch.zeros_like(x), x)


def _frequencies(pairs, scaled):
    """Radians per position, 64 bits.  scaled > 1: pairs that turn less than once in 4096 positions turn that much more slowly,
    those that turn more than 32 times stay, a ramp in between."""
    f = BASE ** (-torch.arange(pairs, dtype=torch.float64, device="cuda") / pairs)
    keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
    return f * (keep + (1 - keep) / scaled)


def prepare(case, seed):
    g = _generator(seed)
    st = {"case": dict(case)}
    if case["op"] == "rotary":
        T, H, D = case["rows"], case["heads"], case["dim"]
        # the q and k heads of a row; v lies behind them
        room = torch.empty(T, H + 2, D, dtype=TYPES[case["type"]], device="cuda")
        room.copy_(torch.randn(T, H + 2, D, generator=g, device="cuda"))
        st["x"] = room[:, :H]
        st["y"] = torch.empty(T, H, D, dtype=room.dtype, device="cuda")
        first = int(torch.randint(0, case["far"], (1,), generator=g, device="cuda"))
        st["positions"] = (first + torch.arange(T, device="cuda")) % case["far"]
        st["frequencies"] = _frequencies(case["pairs"], case["scaled"])
        st["amplitude"] = 1.0 if case["scaled"] == 1.0 else 0.1 * math.log(case["scaled"]) + 1.0
        return st
    Tq, Tk, H, K, D = case["queries"], case["keys"], case["heads"], case["kv_heads"], case["dim"]
    qs, ks = _runs(case)
    st["query_start"] = torch.from_numpy(qs).cuda()
    st["key_start"] = st["query_start"] if ks is qs else torch.from_numpy(ks).cuda()
    # heads of different sharpness, and a first key in every sequence that most queries look at
    common = torch.randn(K, 1, D, generator=g, device="cuda")
    sharp = torch.exp(0.4 * torch.randn(H, 1, generator=g, device="cuda"))
    q = (torch.randn(Tq, K, H // K, D, generator=g, device="cuda") + 0.5 * common).reshape(Tq, H, D) * sharp
    k = torch.randn(Tk, K, D, generator=g, device="cuda")
    firsts = st["key_start"][:-1][st["key_start"][:-1] < Tk]
    k[firsts] += 0.75 * common[:, 0]
    v = torch.randn(Tk, K, D, generator=g, device="cuda") + 0.3
    if ks is qs:
        room = torch.cat([q, k, v], 1).bfloat16()
        st["q"], st["k"], st["v"] = room[:, :H], room[:, H:H + K], room[:, H + K:]
    else:
        room = torch.cat([k, v], 1).bfloat16()
        st["q"], st["k"], st["v"] = q.bfloat16(), room[:, :K], room[:, K:]
    st["y"], st["lse"] = torch.empty(Tq, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(Tq, H, device="cuda")
    if case["op"] == "attention_grad":
        del q, k, v
        # what the forward pass left, a kv head at a time
        see, G = _visible(st), H // K
        for h in range(K):
            part = slice(h * G, (h + 1) * G)
            y, lse = _softmax_of(st["q"][:, part], st["k"][:, h:h + 1], st["v"][:, h:h + 1], see)
            st["y"][:, part], st["lse"][:, part] = y.bfloat16(), lse
        st["dy"] = _gradients(g, Tq, H, D).bfloat16()
        st["dq"] = torch.empty(Tq, H, D, dtype=torch.bfloat16, device="cuda")
        grads = torch.empty(Tk, 2 * K, D, dtype=torch.bfloat16, device="cuda")
        st["dk"], st["dv"] = grads[:, :K], grads[:, K:]
    return st


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _visible(st):
    """[queries][keys]: whether the query sees the key."""
    c = st["case"]
    i, j = torch.arange(c["queries"], device="cuda"), torch.arange(c["keys"], device="cuda")
    sq = torch.searchsorted(st["query_start"][1:].contiguous(), i, right=True)
    sk = torch.searchsorted(st["key_start"][1:].contiguous(), j, right=True)
    see = sq[:, None] == sk
    if c["causal"]:
        # both counted from the end of their sequence
        i, j = i - st["query_start"][1:][sq], j - st["key_start"][1:][sk]
        see &= j <= i[:, None]
        if c["window"]:
            see &= j > i[:, None] - c["window"]
    return see


def _by_kv_head(x, kv_heads):
    """[rows][heads][dim] as [kv_heads][heads of a group * rows][dim] in 32 bits."""
    T, H, D = x.shape
    return x.float().reshape(T, kv_heads, H // kv_heads, D).permute(1, 2, 0, 3).reshape(kv_heads, -1, D)


def _by_row(x, rows):
    """Back to [rows][heads][dim]."""
    K, _, D = x.shape
    return x.reshape(K, -1, rows, D).permute(2, 0, 1, 3).reshape(rows, -1, D)


def _logits(q, k, see):
    """[kv_heads][group][queries][keys], -inf where a key is not seen."""
    K, D = k.shape[1], k.shape[2]
    s = torch.matmul(_by_kv_head(q, K), k.float().permute(1, 2, 0)).view(K, -1, q.shape[0], k.shape[0])
    return s.mul_(1 / math.sqrt(D)).masked_fill_(~see, -math.inf)


def _softmax_of(q, k, v, see):
    T, H, D = q.shape
    s = _logits(q, k, see)
    most = s.amax(3, keepdim=True)
    most = torch.where(most > -math.inf, most, torch.zeros_like(most))
    p = s.sub_(most).exp_()
    total = p.sum(3, keepdim=True)
    lse = (most + total.log()).view(H, T).t().contiguous()
    p = p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    return _by_row(torch.matmul(p.flatten(1, 2), v.float().transpose(0, 1)), T), lse


def _plain(st):
    c = st["case"]
    if c["op"] == "rotary":
        x, n = st["x"].float(), c["pairs"]
        angle = st["positions"].double()[:, None, None] * st["frequencies"]
        cos, sin = (st["amplitude"] * angle.cos()).float(), (st["amplitude"] * angle.sin()).float()
        sin = -sin if c["backward"] else sin
        a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["interleaved"] else (slice(0, n), slice(n, 2 * n))
        y = x.clone()
        y[..., a] = x[..., a] * cos - x[..., b] * sin
        y[..., b] = x[..., a] * sin + x[..., b] * cos
        return {"y": y.to(st["x"].dtype)}
    if c["op"] == "attention":
        y, lse = _softmax_of(st["q"], st["k"], st["v"], _visible(st))
        return {"y": y.bfloat16(), "lse": lse}
    T, K, scale = c["queries"], c["kv_heads"], 1 / math.sqrt(c["dim"])
    lse = torch.where(st["lse"] > -math.inf, st["lse"], torch.zeros_like(st["lse"]))
    p = _logits(st["q"], st["k"], _visible(st)).sub_(lse.t().reshape(K, -1, T, 1)).exp_().flatten(1, 2)
    dy = _by_kv_head(st["dy"], K)
    dv = torch.matmul(p.transpose(1, 2), dy)
    dp = torch.matmul(dy, st["v"].float().permute(1, 2, 0))
    ds = dp.sub_((dy * _by_kv_head(st["y"], K)).sum(2, keepdim=True)).mul_(p)
    dq = scale * torch.matmul(ds, st["k"].float().transpose(0, 1))
    dk = scale * torch.matmul(ds.transpose(1, 2), _by_kv_head(st["q"], K))
    return {"dq": _by_row(dq, T).bfloat16(), "dk": dk.transpose(0, 1).bfloat16(), "dv": dv.transpose(0, 1).bfloat16()}


# ---- the framework's operators -------------------------------------------------------------------------------------

def _framework(st):
    from paper_2103_08870_b200 import layers
    c = st["case"]
    if c["op"] == "rotary":
        layers.rotary(st["x"], st["positions"], st["frequencies"], st["y"], interleaved=c["interleaved"], amplitude=st["amplitude"],
                      backward=c["backward"])
        return {"y": st["y"]}
    runs = {"query_start": st["query_start"], "key_start": st["key_start"]} if c["sequences"] > 1 else {}
    if c["op"] == "attention":
        layers.attention(st["q"], st["k"], st["v"], st["y"], st["lse"], causal=c["causal"], window=c["window"], **runs)
        return {"y": st["y"], "lse": st["lse"]}
    layers.attention_backward(st["dy"], st["q"], st["k"], st["v"], st["y"], st["lse"], st["dq"], st["dk"], st["dv"], causal=c["causal"],
                              window=c["window"], **runs)
    return {"dq": st["dq"], "dk": st["dk"], "dv": st["dv"]}


def run(state):
    return _framework(state) if own else _plain(state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        x, n = st["x"].double(), case["pairs"]
        y = x.clone()
        turn = torch.exp(1j * (-1 if case["backward"] else 1) * st["positions"].double()[:, None] * st["frequencies"][None]) * st["amplitude"]
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + n)
            z = torch.complex(x[:, :, a], x[:, :, b]) * turn[:, i, None]
            y[:, :, a], y[:, :, b] = z.real, z.imag
        return {"y": y}
    Tq, Tk, H, K, D = case["queries"], case["keys"], case["heads"], case["kv_heads"], case["dim"]
    G, (qs, ks) = H // K, _runs(case)
    zeros = lambda *shape: torch.zeros(*shape, dtype=torch.float64, device="cuda")  # noqa: E731
    grad = case["op"] == "attention_grad"
    y, lse = zeros(Tq, H, D), torch.full((Tq, H), -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = zeros(Tq, H, D), zeros(Tk, K, D), zeros(Tk, K, D)
    for s in range(case["sequences"]):
        q0, q1, k0, k1 = int(qs[s]), int(qs[s + 1]), int(ks[s]), int(ks[s + 1])
        if q0 == q1 or k0 == k1:
            continue
        ahead = torch.arange(k0 - k1, 0, device="cuda") - torch.arange(q0 - q1, 0, device="cuda")[:, None]    # of the query's own place
        hidden = torch.zeros_like(ahead, dtype=torch.bool)
        if case["causal"]:
            hidden = (ahead > 0) | ((ahead <= -case["window"]) if case["window"] else hidden)
        for h in range(H):
            q, k, v = st["q"][q0:q1, h].double(), st["k"][k0:k1, h // G].double(), st["v"][k0:k1, h // G].double()
            z = (q @ k.t()) / math.sqrt(D)
            z[hidden] = -math.inf
            if not grad:
                lse[q0:q1, h] = torch.logsumexp(z, 1)
                y[q0:q1, h] = torch.nan_to_num(torch.softmax(z, 1)) @ v
                continue
            known = st["lse"][q0:q1, h, None].double()
            p = torch.where(hidden, torch.zeros_like(z), torch.exp(z - known))
            dy = st["dy"][q0:q1, h].double()
            dz = p * (dy @ v.t() - (dy * st["y"][q0:q1, h].double()).sum(1, keepdim=True))
            dq[q0:q1, h] = dz @ k / math.sqrt(D)
            dk[k0:k1, h // G] += dz.t() @ q / math.sqrt(D)
            dv[k0:k1, h // G] += p.t() @ dy
    return {"dq": dq, "dk": dk, "dv": dv} if grad else {"y": y, "lse": lse}
