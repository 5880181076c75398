"""Timed work of the operators around the embedding layer's rows: dropout from
a counter-based generator, layer norm (forward and backward, with the dropout
and the residual of the layer before it) and the learned relative position
bias by buckets (forward and gradient).

`own` false: the operators in their plain form (elementary torch operations in
float32).  `own` true: the calls that a program makes of the layer's binding.
A case is a dict of plain values:

  op        "dropout", "norm", "norm_grad", "bias" or "bias_grad"
  rows, cols, pad      rows of `cols` elements, `pad` elements apart from the
                       next row (a view of wider rows)
  dtype     "f32" or "bf16": rows, scores and their gradients
  wtype     the same for the learned weights (norm weight and bias, bias table)
  p         dropout probability (0: none)
  residual  a residual is added (norm, norm_grad: and its sum is kept)
  B, H, Q, K           batch, heads, queries, keys of the scores
  buckets, far, both   buckets, the distance of the last one, whether keys
                       behind and ahead of the query have buckets of their own
  start     position of the first query; -1: one per sequence, on the GPU
  scores    the bias is added to scores (else it is written alone)
"""
import math

import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MASK32 = 0xFFFFFFFF


def _rows(name, op, rows, cols, dtype, *, wtype="f32", p=0.0, residual=False, pad=0):
    c = dict(op=op, rows=rows, cols=cols, dtype=dtype, wtype=wtype, p=p, residual=residual, pad=pad)
    return dict(c, name=name) if name else c


def _bias(name, op, B, H, Q, K, dtype, *, wtype="f32", buckets=32, far=128, both=True, start=0,
          scores=True):
    c = dict(op=op, B=B, H=H, Q=Q, K=K, dtype=dtype, wtype=wtype, buckets=buckets, far=far,
             both=both, start=start, scores=scores)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short sequence's rows, odd width, a view of wider rows
        _rows("drop_few_odd", "dropout", 37, 1001, "f32", p=0.1, residual=True, pad=23),
        # pooled rows of a batch of 16384 samples and 26 tables, as a whole
        _rows("drop_pooled_rows", "dropout", 16384, 26 * 128, "f32", p=0.2),
        # a layer's output onto its residual stream, a large training batch
        _rows("drop_residual_bf16", "dropout", 32768, 4096, "bf16", p=0.1, residual=True),
        # one token being answered
        _rows("norm_one_token", "norm", 1, 4096, "bf16", wtype="bf16"),
        # every table's embedding of 16384 samples normalised on its own
        _rows("norm_tables_f32", "norm", 16384 * 26, 128, "f32"),
        # residual + dropout + norm of a training batch
        _rows("norm_add_drop_bf16", "norm", 16384, 4096, "bf16", p=0.1, residual=True),
        # gradient of the tables' norm at batch 2048
        _rows("norm_grad_tables", "norm_grad", 2048 * 26, 128, "f32"),
        # gradient of residual + dropout + norm of a training batch
        _rows("norm_grad_add_drop", "norm_grad", 16384, 4096, "bf16", p=0.1, residual=True),
        # one new token of each of 64 sequences, every one at its own length
        _bias("bias_next_token", "bias", 64, 16, 1, 4096, "bf16", both=False, start=-1),
        # scores of whole prompts
        _bias("bias_prompt", "bias", 4, 16, 2048, 2048, "bf16"),
        # gradient of the table, small odd sequences of a causal model
        _bias("bias_grad_odd", "bias_grad", 3, 5, 131, 517, "f32", both=False, start=386),
        # gradient of the table over whole prompts
        _bias("bias_grad_prompt", "bias_grad", 4, 16, 2048, 2048, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["dropout", "norm", "norm_grad", "bias", "bias_grad"])
    dtype, wtype = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    if op in ("dropout", "norm", "norm_grad"):
        cols = _log(rng, 1, 16384)
        if rng.random() < 0.5:
            cols = max(8, cols // 8 * 8)
        rows = _log(rng, 1, min(65536, (1 << (26 if dtype == "bf16" else 25)) // cols))
        return _rows(None, op, rows, cols, dtype, wtype=wtype,
                     p=rng.choice([0.05, 0.1, 0.5]) if op == "dropout" or rng.random() < 0.5 else 0.0,
                     residual=rng.random() < 0.5, pad=rng.choice([0, 0, 8, 5]))
    both = rng.random() < 0.5
    buckets = rng.choice([8, 16, 32, 64])
    far = rng.choice([64, 128, 250, 1000])
    H = _log(rng, 1, 32)
    B = _log(rng, 1, 64)
    if rng.random() < 0.3:
        Q, K = 1, _log(rng, 1, 32768)
    else:
        Q = _log(rng, 1, 2048)
        K = rng.choice([Q, Q + _log(rng, 1, 4096)])
    while B * H * Q * K > (1 << 27) - (1 << 20):
        B, H = max(1, B // 2), (max(1, H // 2) if B == 1 else H)
    return _bias(None, op, B, H, Q, K, dtype, wtype=wtype, buckets=buckets, far=far, both=both,
                 start=rng.choice([0, K - Q, -1]), scores=op == "bias_grad" or rng.random() < 0.8)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------


def _inputs(case, seed):
    """The data of a case, from the seed alone."""
    g = torch.Generator("cuda").manual_seed(seed)
    dt, wt = TYPES[case["dtype"]], TYPES[case["wtype"]]

    def normal(shape, scale=1.0, to=dt):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(to)

    s = {"case": case}
    if "rows" in case:
        R, C, pad = case["rows"], case["cols"], case["pad"]

        def rows(scale=1.0, shift=0.0):
            wide = normal((R, C + pad), scale, torch.float32).add_(shift).to(dt)
            return wide[:, :C]

        # key and number of the mask
        s["seed"] = int(torch.randint(0, 2**62, (), generator=g, device="cuda").item())
        s["offset"] = int(torch.randint(0, 2**40, (), generator=g, device="cuda").item())
        if case["op"] == "norm_grad":
            s["x"] = rows(1.5, 0.3)  # the sum that was normalised
            x = s["x"].double()
            mean = x.mean(1)
            s["mean"] = mean.float()
            s["rstd"] = ((x - mean[:, None]).pow(2).mean(1) + EPS).rsqrt().float()
            s["grad"] = rows(1e-2)
            s["grad_sum"] = rows(1e-2) if case["residual"] else None
        else:
            s["x"] = rows(1.5, 0.3)
            s["residual"] = rows(1.0, -0.1) if case["residual"] else None
        if case["op"] != "dropout":
            s["weight"] = (1 + normal((C,), 0.1, torch.float32)).to(wt)
            s["bias"] = normal((C,), 0.1, wt)
        return s
    B, H, Q, K = (case[k] for k in "BHQK")
    s["table"] = normal((case["buckets"], H), 0.5, wt)
    s["starts"] = None
    if case["start"] < 0:  # every sequence has its own length
        s["starts"] = torch.randint(0, max(1, K), (B,), generator=g, device="cuda",
                                    dtype=torch.int32)
    if case["scores"]:
        x = normal((B, H, Q, K), 2.0 if case["op"] == "bias" else 1e-2)
        if not case["both"]:  # causal: nothing behind the query's position is seen
            q = torch.arange(Q, device="cuda") + max(0, case["start"])
            ahead = torch.arange(K, device="cuda")[None, :] > q[:, None]
            if case["start"] >= 0:
                x.masked_fill_(ahead, -math.inf if case["op"] == "bias" else 0.0)
        s["x"] = x
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        if "rows" not in case:
            s["borders"] = torch.tensor(_borders(case), device="cuda")
        return s
    # what a program keeps: parameter blocks and the buffers of the results
    from paper_2207_10731_amd import pss
    s["pss"] = pss
    dt = TYPES[case["dtype"]]
    if "rows" in case:
        R, C = case["rows"], case["cols"]
        s["drop"] = (pss.make_dropout_params(case["p"], s["seed"], s["offset"])
                     if case["p"] > 0 else None)
        s["out"] = torch.empty((R, C), dtype=dt, device="cuda")
        if case["op"] == "norm":
            s["mean"], s["rstd"] = (torch.empty(R, device="cuda") for _ in range(2))
            s["sum"] = torch.empty((R, C), dtype=dt, device="cuda") if case["residual"] else None
        if case["op"] == "norm_grad":
            s["gw"], s["gb"] = (torch.empty(C, device="cuda") for _ in range(2))
            s["gres"] = (torch.empty((R, C), dtype=dt, device="cuda")
                         if case["residual"] and case["p"] > 0 else None)
        return s
    s["map"] = pss.make_position_buckets(case["buckets"], case["far"], case["both"])
    if case["op"] == "bias":
        s["out"] = torch.empty(tuple(case[k] for k in "BHQK"), dtype=dt, device="cuda")
    else:
        s["gt"] = torch.empty((case["buckets"], case["H"]), device="cuda")
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------


def run(state):
    return (_own if own else _plain)(state)


def _own(s):
    c, pss = s["case"], s["pss"]
    op = c["op"]
    if op == "dropout":
        return pss.pss_dropout(s["x"], s["drop"], s["out"], residual=s["residual"])
    if op == "norm":
        pss.pss_layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, s["out"], s["mean"],
                                   s["rstd"], residual=s["residual"], dropout=s["drop"],
                                   sum_out=s["sum"])
        return [t for t in (s["out"], s["mean"], s["rstd"], s["sum"]) if t is not None]
    if op == "norm_grad":
        pss.pss_layer_norm_backward(s["grad"], s["x"], s["weight"], s["mean"], s["rstd"], s["out"],
                                    s["gw"], s["gb"], grad_sum=s["grad_sum"], dropout=s["drop"],
                                    grad_residual=s["gres"])
        return [t for t in (s["out"], s["gw"], s["gb"], s["gres"]) if t is not None]
    if op == "bias":
        return pss.pss_position_bias_forward(s["table"], s["map"], s["out"], scores=s.get("x"),
                                             q_start=max(0, c["start"]), q_starts=s["starts"])
    return pss.pss_position_bias_backward(s["x"], s["map"], s["gt"], q_start=max(0, c["start"]),
                                          q_starts=s["starts"])


def _kept(p, seed, offset, R, C):
    """Factor of every element: 0 or the inverse of the share kept.  Element
    (r, c) is one of the eight 16-bit numbers of Philox4x32-10 (Salmon et al.
    2011) at counter (c / 8, r, offset) and key `seed`; it is dropped when its
    number lies below the probability in units of 2^-16."""
    n = (C + 7) // 8
    c0 = torch.arange(n, device="cuda").expand(R, n)
    c1 = torch.arange(R, device="cuda")[:, None].expand(R, n)
    c2 = torch.full((R, n), offset & MASK32, device="cuda")
    c3 = torch.full((R, n), offset >> 32, device="cuda")
    k0, k1 = seed & MASK32, seed >> 32
    for _ in range(10):
        lo0, lo1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        hi0, hi1 = (lo0 >> 32) & MASK32, (lo1 >> 32) & MASK32
        c0, c1, c2, c3 = (hi1 ^ c1 ^ k0), lo1 & MASK32, (hi0 ^ c3 ^ k1), lo0 & MASK32
        k0, k1 = (k0 + 0x9E3779B9) & MASK32, (k1 + 0xBB67AE85) & MASK32
    words = torch.stack([c0, c1, c2, c3], -1)
    numbers = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(R, n * 8)[:, :C]
    t = int(math.floor(p * 65536 + 0.5))
    return (numbers >= t).float() * (65536 / (65536 - t) if t < 65536 else 0.0)


def _plain(s):
    c = s["case"]
    op, dt = c["op"], TYPES[c["dtype"]]
    if "rows" in c:
        R, C = c["rows"], c["cols"]
        kept = _kept(c["p"], s["seed"], s["offset"], R, C) if c["p"] > 0 else None
    if op in ("dropout", "norm"):
        x = s["x"].float()
        if kept is not None:
            x = x * kept
        if s["residual"] is not None:
            x = x + s["residual"].float()
        if op == "dropout":
            return x.to(dt)
        mean = x.sum(1, keepdim=True) / C
        away = x - mean
        rstd = 1 / torch.sqrt((away * away).sum(1, keepdim=True) / C + EPS)
        y = away * rstd * s["weight"].float() + s["bias"].float()
        out = [y.to(dt), mean[:, 0], rstd[:, 0]]
        return out + [x.to(dt)] if s["residual"] is not None else out
    if op == "norm_grad":
        rstd = s["rstd"][:, None]
        xhat = (s["x"].float() - s["mean"][:, None]) * rstd
        dy = s["grad"].float()
        gw, gb = (dy * xhat).sum(0), dy.sum(0)
        h = dy * s["weight"].float()
        dx = (h - h.sum(1, keepdim=True) / C - xhat * ((h * xhat).sum(1, keepdim=True) / C)) * rstd
        if s["grad_sum"] is not None:
            dx = dx + s["grad_sum"].float()
        through = dx if kept is None else dx * kept
        out = [through.to(dt), gw, gb]
        return out + [dx.to(dt)] if c["residual"] and kept is not None else out
    B, H, Q, K = (c[k] for k in "BHQK")
    first = torch.full((B,), max(0, c["start"]), device="cuda")
    if s["starts"] is not None:
        first = first + s["starts"]
    else:
        first = first[:1]  # the same for every sequence
    away = torch.arange(K, device="cuda") - (first[:, None, None] + torch.arange(Q, device="cuda")[:, None])
    far = away.abs() if c["both"] else (-away).clamp(min=0)
    bucket = torch.zeros_like(far)
    for b in s["borders"][1:]:
        bucket += far >= b
    if c["both"]:
        bucket += (away > 0) * (c["buckets"] // 2)
    if op == "bias":
        out = s["table"].float()[bucket].permute(0, 3, 1, 2)
        out = out + s["x"].float() if c["scores"] else out.expand(B, H, Q, K)
        return out.to(dt).contiguous()
    g = s["x"].float()
    return torch.stack([(g * (bucket == n).float()[:, None]).sum((0, 2, 3))
                        for n in range(c["buckets"])])


def _borders(case):
    """Smallest distance of every bucket of one side: e distances of their
    own, then the first n with n^L >= e^(L-j) * far^j (the logarithm's steps)."""
    side = case["buckets"] // 2 if case["both"] else case["buckets"]
    e = side // 2
    L = side - e
    out = list(range(e))
    for j in range(L):
        want = e ** (L - j) * case["far"] ** j
        n = int(e * (case["far"] / e) ** (j / L))
        while n > 0 and (n - 1) ** L >= want:
            n -= 1
        while n ** L < want:
            n += 1
        out.append(n)
    return out


# ---------------------------------------------------------------------------
# From the definitions, in 64 bits
# ---------------------------------------------------------------------------


def _exact_kept(p, seed, offset, R, C):
    """The mask again, from the generator's definition with products in
    16-bit halves."""
    n = -(-C // 8)

    def product(a, x):
        a0, a1, x0, x1 = a & 0xFFFF, a >> 16, x & 0xFFFF, x >> 16
        low = a0 * x0
        mid = a1 * x0 + (low >> 16)
        mid2 = a0 * x1 + (mid & 0xFFFF)
        return a1 * x1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | (low & 0xFFFF)

    at = torch.arange(R * n, device="cuda")
    x = [at % n, at // n, torch.full_like(at, offset % 2**32), torch.full_like(at, offset // 2**32)]
    key = [seed % 2**32, seed // 2**32]
    for turn in range(10):
        h, l = product(0xD2511F53, x[0])
        h2, l2 = product(0xCD9E8D57, x[2])
        keys = ((key[0] + turn * 0x9E3779B9) % 2**32, (key[1] + turn * 0xBB67AE85) % 2**32)
        x = [h2 ^ x[1] ^ keys[0], l2, h ^ x[3] ^ keys[1], l]
    u = torch.empty((R, n, 8), dtype=torch.int32, device="cuda")
    for k in range(8):
        u[:, :, k] = ((x[k // 2] >> (16 * (k % 2))) % 65536).view(R, n)
    limit = round(p * 65536)
    keep = (u.view(R, n * 8)[:, :C] >= limit).double()
    return keep.mul_(65536 / (65536 - limit))


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("dropout", "norm"):
        v = s["x"].double()
        if case["p"] > 0:
            v = v * _exact_kept(case["p"], s["seed"], s["offset"], case["rows"], case["cols"])
        if case["residual"]:
            v = v + s["residual"].double()
        if op == "dropout":
            return v
        var, mean = torch.var_mean(v, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(s["bias"].double(), (v - mean[:, None]) * rstd[:, None], s["weight"].double())
        return [y, mean, rstd] + ([v] if case["residual"] else [])
    if op == "norm_grad":
        C = case["cols"]
        r = s["rstd"].double()[:, None]
        z = (s["x"].double() - s["mean"].double()[:, None]) * r
        dy = s["grad"].double()
        dz = dy * s["weight"].double()
        # the transposed Jacobian of the normalisation: r (I - 1 1'/C - z z'/C)
        dv = r * (dz - dz.mean(1, keepdim=True) - z * torch.linalg.vecdot(dz, z)[:, None] / C)
        if case["residual"]:
            dv = dv + s["grad_sum"].double()
        gw, gb = (dy * z).sum(0), dy.sum(0)
        if case["p"] == 0:
            return [dv, gw, gb]
        keep = _exact_kept(case["p"], s["seed"], s["offset"], case["rows"], C)
        return [dv * keep, gw, gb] + ([dv] if case["residual"] else [])
    B, H, Q, K = (case[k] for k in "BHQK")
    side = case["buckets"] // (2 if case["both"] else 1)
    e = side // 2
    # bucket of every distance -(K + Q) .. K + Q, by the logarithm (a distance
    # on a border differs from the border by its rounding alone)
    start = max(0, case["start"])
    reach = K + Q + start + (K if case["start"] < 0 else 0) + 1
    away = torch.arange(-reach, reach + 1, dtype=torch.float64)
    n = away.abs() if case["both"] else (-away).clamp(min=0)
    step = (n.clamp(min=1) / e).log() / math.log(case["far"] / e) * (side - e)
    by_log = e + (step + 1e-9).floor().clamp(max=side - 1 - e)
    of = torch.where(n < e, n, by_log).long()
    if case["both"]:
        of = of + (away > 0).long() * side
    of = of.cuda()
    table, x = s["table"].double(), s.get("x")
    out = torch.zeros((case["buckets"], H), dtype=torch.float64, device="cuda")
    full = torch.empty((B, H, Q, K), dtype=torch.float64, device="cuda") if op == "bias" else None
    for b in range(B):
        at = start + (int(s["starts"][b]) if s["starts"] is not None else 0)
        q = torch.arange(at, at + Q, device="cuda")
        bucket = of[torch.arange(K, device="cuda")[None, :] - q[:, None] + reach]
        for h in range(H):
            if op == "bias":
                full[b, h] = table[:, h][bucket]
                if case["scores"]:
                    full[b, h] += x[b, h].double()
            else:
                out[:, h].scatter_add_(0, bucket.reshape(-1), x[b, h].double().reshape(-1))
    return full if op == "bias" else out


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------


def work(case):
    size = {"f32": 4, "bf16": 2}
    e, w = size[case["dtype"]], size[case["wtype"]]
    if "rows" in case:
        n, C, R = case["rows"] * case["cols"], case["cols"], case["rows"]
        res = case["residual"]
        if case["op"] == "dropout":
            return {"bytes": n * e * (3 if res else 2), "flops": n * (2 if res else 1)}
        if case["op"] == "norm":
            return {"bytes": n * e * (4 if res else 2) + 2 * C * w + 8 * R, "flops": 9 * n}
        both = res and case["p"] > 0
        return {"bytes": n * e * (3 + res + both) + C * w + 8 * C + 8 * R, "flops": 14 * n}
    n = case["B"] * case["H"] * case["Q"] * case["K"]
    if case["op"] == "bias":
        return {"bytes": n * e * (2 if case["scores"] else 1) + case["buckets"] * case["H"] * w,
                "flops": n}
    return {"bytes": n * e + case["buckets"] * case["H"] * 4, "flops": n}
