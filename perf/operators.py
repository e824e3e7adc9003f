"""The operators around a training step whose loss is this library's, as measurable cases.

An encoder that moves point sets is trained on the gradient of the Sinkhorn loss.  What it computes besides matrix products:

  attention  softmax attention over the points of a set, forward (``Context.fs_attention``): training's forward pass, inference,
             and single queries over a long cache of keys
  train      its forward and its backward pass (``Context.fs_attention_grad``), which recomputes the probabilities
  norm       layer norm, forward and backward, with the gradients of its weights (``fs_layer_norm``, ``fs_layer_norm_grad``)
  adamw      one optimiser step over all weights at once (``binding.AdamW``), its state in 32 or in 8 bits

Each has a plain form here: elementary torch operations in 32 bits, rounded once to the type of the output.
"""
from __future__ import annotations

import math

import torch

own = False   # True: the library's entry points instead of the plain forms

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BLOCK = 256   # weights that share a scale of an 8-bit state

# What each listed case stands for:
#  points_1024_d64      inference on a batch of the benchmark's smallest point sets: little work, bound by the launch
#  points_16k_d64       one set of the transport workload's size (16384 points) through sixteen heads
#  query_50k_d128       one new query for each of four sets over a cache of some 50000 keys, eight kv heads shared by four each
#  train_1024_d64       a training batch of small sets, q, k and v as one projection wrote them
#  train_ragged_f32     sets of unequal sizes with weights (log-weights as bias, some points removed), odd sizes, full precision
#  train_8k_d128        a long ordered sequence: every point sees those before it, kv heads shared by four
#  norm_1024_d64        the smallest norm, bound by its launches
#  norm_70k_d784        image-shaped rows in full precision
#  norm_50k_d1024       embedding rows in bf16
#  adamw_64_f32         the weights of a narrow encoder: many small tensors, full precision
#  adamw_784_f32        an encoder as wide as the images, state in 32 bits
#  adamw_1024_8bit      a wide encoder: bf16 weights and gradients with float masters, state in 8 bits
_LISTED = [
    dict(name="points_1024_d64", op="attention", dtype="bf16", batch=4, n=1024, m=1024, heads=4, kv_heads=4, d=64, causal=False,
         ragged=False, bias=False, packed=True),
    dict(name="points_16k_d64", op="attention", dtype="bf16", batch=1, n=16384, m=16384, heads=16, kv_heads=16, d=64, causal=False,
         ragged=False, bias=False, packed=True),
    dict(name="query_50k_d128", op="attention", dtype="bf16", batch=4, n=1, m=50021, heads=32, kv_heads=8, d=128, causal=False,
         ragged=True, bias=False, packed=False),
    dict(name="train_1024_d64", op="train", dtype="bf16", batch=8, n=1024, m=1024, heads=8, kv_heads=8, d=64, causal=False,
         ragged=False, bias=False, packed=True),
    dict(name="train_ragged_f32", op="train", dtype="f32", batch=3, n=1000, m=777, heads=4, kv_heads=4, d=40, causal=False,
         ragged=True, bias=True, packed=False),
    dict(name="train_8k_d128", op="train", dtype="bf16", batch=1, n=8192, m=8192, heads=16, kv_heads=4, d=128, causal=True,
         ragged=False, bias=False, packed=False),
    dict(name="norm_1024_d64", op="norm", dtype="bf16", rows=1024, cols=64, ld=64),
    dict(name="norm_70k_d784", op="norm", dtype="f32", rows=70000, cols=784, ld=784),
    dict(name="norm_50k_d1024", op="norm", dtype="bf16", rows=50000, cols=1024, ld=1024),
    dict(name="adamw_64_f32", op="adamw", dtype="f32", layers=6, width=64, inner=256, points=3, bits=32, master=False),
    dict(name="adamw_784_f32", op="adamw", dtype="f32", layers=4, width=784, inner=3136, points=784, bits=32, master=False),
    dict(name="adamw_1024_8bit", op="adamw", dtype="bf16", layers=8, width=1024, inner=4096, points=64, bits=8, master=True),
]


def listed():
    return [dict(c) for c in _LISTED]


def _log(rng, lo, hi):
    """A whole number spread evenly over its logarithm."""
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "train", "train", "norm", "adamw"])
    if op == "norm":
        cols = _log(rng, 16, 8192)
        rows = _log(rng, 1, min(70000, 60_000_000 // cols))
        return dict(op=op, dtype=rng.choice(["f32", "bf16"]), rows=rows, cols=cols, ld=cols + rng.choice([0, 0, 8, 3]))
    if op == "adamw":
        width = _log(rng, 16, 1024)
        dtype = rng.choice(["f32", "bf16"])
        return dict(op=op, dtype=dtype, layers=rng.randint(1, 8), width=width, inner=width * rng.choice([1, 2, 4]),
                    points=_log(rng, 2, 1024), bits=rng.choice([8, 32]), master=dtype == "bf16" and rng.random() < 0.7)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([32, 40, 64, 64, 80, 96, 128, 128, rng.randint(8, 128)])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 4])
    batch = rng.choice([1, 2, 3, 8])
    same = rng.random() < 0.5
    m = _log(rng, 16, 50021)
    n = m if same else rng.choice([1, _log(rng, 1, 16384)])
    most = (1.0e12 if dtype == "bf16" else 1.0e11) / (4 if op == "attention" else 14) / d   # score entries
    most = min(most, 3.0e9)
    while batch * heads * n * m > most:   # (by the longer side, so that short queries over long keys stay)
        if n >= m:
            n = max(1, n // 2)
            m = n if same else m
        else:
            m = max(1, m // 2)
    packed = same and heads == kv_heads and rng.random() < 0.5
    return dict(op=op, dtype=dtype, batch=batch, n=n, m=m, heads=heads, kv_heads=kv_heads, d=d, causal=same and rng.random() < 0.5,
                ragged=rng.random() < 0.4, bias=rng.random() < 0.3, packed=packed)


# ---- inputs --------------------------------------------------------------------------------------------

def _lengths(case):
    """Points of each set: the first is whole, the others are shorter by even steps."""
    b, m = case["batch"], case["m"]
    return [m - (m * i) // (2 * b) for i in range(b)] if case["ragged"] else [m] * b


def _shapes(case):
    """The weights of an encoder: embedding, layers of two norms, four attention maps and two inner maps, output."""
    w, i = case["width"], case["inner"]
    one = [(w,), (w,), (3 * w, w), (3 * w,), (w, w), (w,), (w,), (w,), (i, w), (i,), (w, i), (w,)]
    return [(w, case["points"]), (w,)] + one * case["layers"] + [(case["points"], w), (case["points"],)]


def _padded(case):
    return sum(-(-math.prod(s) // _BLOCK) * _BLOCK for s in _shapes(case))


def _views(flat, case):
    """The tensors inside a flat buffer: each starts at a whole block."""
    at, got = 0, []
    for s in _shapes(case):
        n = math.prod(s)
        got.append(flat[at:at + n])
        at += -(-n // _BLOCK) * _BLOCK
    return got


def _inside(case, device):
    """1 where the flat buffer holds a weight, 0 in the padding."""
    keep = torch.zeros(_padded(case), device=device)
    torch._foreach_add_(_views(keep, case), 1.0)
    return keep


def _context():
    from paper_2602_03067_amd import binding
    return binding.Context(0)


def _attention_inputs(case, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    dt = _TYPES[case["dtype"]]
    b, n, m, h, hk, d = (case[k] for k in ("batch", "n", "m", "heads", "kv_heads", "d"))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda:0").to(dt)

    if case["packed"]:
        q, k, v = normal(b, n, 3, h, d).unbind(2)
    else:
        q, k, v = normal(b, n, h, d), normal(b, m, hk, d), normal(b, m, hk, d)
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda:0") if case["ragged"] else None
    bias = None
    if case["bias"]:   # log-weights of the points, a tenth of them removed
        w = torch.rand(b, m, generator=g, device="cuda:0") + 0.25
        gone = torch.rand(b, m, generator=g, device="cuda:0") < 0.1
        bias = torch.where(gone, torch.full_like(w, -math.inf), torch.log(w))
    state = dict(q=q, k=k, v=v, k_len=lens, bias=bias, causal=case["causal"], scale=1.0 / math.sqrt(d))
    if case["op"] == "train":
        state["do"] = normal(b, n, h, d)
    return state


def _norm_inputs(case, seed):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    dt, r, c = _TYPES[case["dtype"]], case["rows"], case["cols"]
    x = (torch.randn(r, case["ld"], generator=g, device="cuda:0") * 2.0 + 0.5).to(dt)[:, :c]
    dy = torch.randn(r, case["ld"], generator=g, device="cuda:0").to(dt)[:, :c]
    gamma = 1.0 + 0.1 * torch.randn(c, generator=g, device="cuda:0")
    beta = 0.1 * torch.randn(c, generator=g, device="cuda:0")
    return dict(x=x, dy=dy, gamma=gamma, beta=beta, eps=1e-5)


def _adamw_inputs(case, seed):
    """The middle of a training run: weights, gradients, and a state that fits them."""
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    n, dt = _padded(case), _TYPES[case["dtype"]]
    keep = _inside(case, "cuda:0")
    p = torch.randn(n, generator=g, device="cuda:0") * 0.02 * keep
    grad = torch.randn(n, generator=g, device="cuda:0") * 1e-3 * keep
    m = torch.randn(n, generator=g, device="cuda:0") * 3e-4 * keep
    root = (0.5 + torch.rand(n, generator=g, device="cuda:0")) * 1e-3 * keep
    state = dict(p=p.to(dt), grad=grad.to(dt), master=p if case["master"] else None, step=100 + seed % 1000, bits=case["bits"],
                 lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
    if case["bits"] == 8:
        state["m"], state["m_scale"] = _to_8bit(m, _dither(n, 1, "cuda:0") & 0xFFFF)
        state["v"], state["v_scale"] = _to_8bit(root, _dither(n, 1, "cuda:0") >> 16)
    else:
        state["m"], state["v"] = m, root * root
    return state


def prepare(case, seed):
    state = {"attention": _attention_inputs, "train": _attention_inputs, "norm": _norm_inputs, "adamw": _adamw_inputs}[case["op"]](case, seed)
    state["op"] = case["op"]
    if own:
        state["ctx"] = _context()
        if case["op"] == "adamw":
            from paper_2602_03067_amd import binding
            lists = {k: _views(state[k], case) if state.get(k) is not None else None for k in ("p", "grad", "master", "m", "v")}
            blocks = [-(-math.prod(s) // _BLOCK) for s in _shapes(case)]
            for k in ("m_scale", "v_scale"):
                lists[k] = list(torch.split(state[k], blocks)) if k in state else None
            state["grads"] = lists["grad"]
            state["adamw"] = binding.AdamW(state["ctx"], lists["p"], lr=state["lr"], betas=state["betas"], eps=state["eps"],
                                           weight_decay=state["weight_decay"], state_bits=case["bits"], master=lists["master"],
                                           m=lists["m"], v=lists["v"], m_scale=lists["m_scale"], v_scale=lists["v_scale"], step=state["step"])
    return state


# ---- plain forms ---------------------------------------------------------------------------------------

def _plain_forward(s):
    """Softmax attention: o, the largest score of each row and its sum of exponentials, and what the backward pass takes up."""
    q, k, v = (s[x].float().permute(0, 2, 1, 3).contiguous() for x in ("q", "k", "v"))
    (b, h, n, d), hk, m = q.shape, k.shape[1], k.shape[2]
    q = q.reshape(b, hk, (h // hk) * n, d)   # queries of the heads that share keys, one after the other
    sc = (q @ k.transpose(-1, -2)).reshape(b, h, n, m)
    sc *= s["scale"]
    if s["bias"] is not None:
        sc += s["bias"].view(b, 1, 1, m)
    col = torch.arange(m, device=q.device).view(1, 1, 1, m)
    if s["k_len"] is not None:
        sc.masked_fill_(col >= s["k_len"].view(b, 1, 1, 1), -math.inf)
    if s["causal"]:   # the last query sees the last key of its set
        last = (s["k_len"].view(b, 1, 1, 1) if s["k_len"] is not None else m) - n
        sc.masked_fill_(col > torch.arange(n, device=q.device).view(1, 1, n, 1) + last, -math.inf)
    top = sc.amax(-1, keepdim=True)
    sc -= torch.where(top == -math.inf, torch.zeros_like(top), top)
    pr = sc.exp_()
    total = pr.sum(-1, keepdim=True)
    o = (pr.reshape(b, hk, -1, m) @ v).reshape(b, h, n, d) / torch.where(total == 0, torch.ones_like(total), total)
    return o, torch.cat([top, total], -1), (q, k, v, pr, total)


def _plain_attention(s):
    o, stat, _ = _plain_forward(s)
    return {"o": o.permute(0, 2, 1, 3).to(s["q"].dtype), "stat": stat}


def _plain_train(s):
    o, stat, (q, k, v, pr, total) = _plain_forward(s)
    dt = s["q"].dtype
    b, h, n, d = o.shape
    hk, m = k.shape[1], k.shape[2]
    do = s["do"].float().permute(0, 2, 1, 3).contiguous()
    pr /= torch.where(total == 0, torch.ones_like(total), total)
    dv = pr.reshape(b, hk, -1, m).transpose(-1, -2) @ do.reshape(b, hk, -1, d)
    ds = (do.reshape(b, hk, -1, d) @ v.transpose(-1, -2)).reshape(b, h, n, m)
    ds -= (do * o).sum(-1, keepdim=True)
    ds *= pr
    rows = ds.reshape(b, hk, -1, m)
    dq = (rows @ k).reshape(b, h, n, d) * s["scale"]
    dk = (rows.transpose(-1, -2) @ q) * s["scale"]
    out = {"o": o, "dq": dq, "dk": dk, "dv": dv}
    out = {x: t.permute(0, 2, 1, 3).to(dt) for x, t in out.items()}
    out["stat"] = stat
    if s["bias"] is not None:
        out["dbias"] = ds.sum((1, 2)).to(dt)
    return out


def _plain_norm(s):
    x, dy, dt = s["x"].float(), s["dy"].float(), s["x"].dtype
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + s["eps"])
    xh = xc * rstd
    y = xh * s["gamma"] + s["beta"]
    w = dy * s["gamma"]
    dx = rstd * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
    return {"y": y.to(dt), "stat": torch.cat([mean, rstd], 1), "dx": dx.to(dt), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _dither(n, seed, device):
    """32 bits for each weight from its number and the step's seed: the lower half dithers m, the upper half the root of v."""
    at = torch.arange(n, device=device, dtype=torch.int64)
    h = ((at * 0x9E3779B1) & 0xFFFFFFFF) ^ ((seed * 0xB7E15163) & 0xFFFFFFFF)
    h = ((h ^ (h >> 16)) * 0x85A308D3) & 0xFFFFFFFF
    h = ((h ^ (h >> 13)) * 0xB7E15163) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _to_8bit(x, half):
    """8-bit floats (four bits of exponent, three of mantissa) under a power of two for each block, rounded up or down by the dither:
    the largest of a block lies in (224, 448] of its scale."""
    x = x.view(-1, _BLOCK)
    top = x.abs().amax(1, keepdim=True)
    frac, e = torch.frexp(top)
    scale = ((torch.clamp(torch.where(frac > 0.875, e - 8, e - 9), -100, 100) + 127) << 23).to(torch.int32).view(torch.float32)
    scale = torch.where(top == 0, torch.ones_like(top), scale)
    a = (x.abs() / scale).contiguous()
    low = ((half.view(-1, _BLOCK) << 4) | 8).to(torch.int32)   # twenty bits: as many as are dropped
    normal = ((a.view(torch.int32) + low) >> 20) - (120 << 3)
    small = torch.floor(a * 512.0 + low.float() * 2.0 ** -20).to(torch.int32)
    code = torch.where(a >= 2.0 ** -6, normal, small) | torch.where(x < 0, 128, 0).to(torch.int32)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).reshape(-1), scale.reshape(-1)


def _from_8bit(code, scale):
    return (code.float().view(-1, _BLOCK) * scale.view(-1, 1)).reshape(-1)


def _plain_adamw(s):
    s["step"] += 1
    (b1, b2), t = s["betas"], s["step"]
    p = s["master"] if s["master"] is not None else s["p"].float()
    g = s["grad"].float()
    if s["bits"] == 8:
        m, root = _from_8bit(s["m"], s["m_scale"]), _from_8bit(s["v"], s["v_scale"])
        v = root * root
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    root = torch.sqrt(v)
    p = p * (1 - s["lr"] * s["weight_decay"]) - (s["lr"] / (1 - b1 ** t)) * m / (root * (1 / math.sqrt(1 - b2 ** t)) + s["eps"])
    out = {}
    if s["bits"] == 8:
        h = _dither(p.numel(), t, p.device)
        m, s["m_scale"] = _to_8bit(m, h & 0xFFFF)
        code, s["v_scale"] = _to_8bit(root, h >> 16)
        code = torch.where((code.view(torch.uint8) == 0) & (root > 0), 1, code.view(torch.uint8))   # a root above zero stays above it
        v = code.view(torch.float8_e4m3fn)
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    if s["master"] is not None:
        s["master"] = p
        out["master"] = p
    s["m"], s["v"], s["p"] = m, v, p.to(s["p"].dtype)
    out.update(p=s["p"], m=m, v=v)
    return out


def run(state):
    if not own:
        return {"attention": _plain_attention, "train": _plain_train, "norm": _plain_norm, "adamw": _plain_adamw}[state["op"]](state)
    s, ctx = state, state["ctx"]
    if s["op"] in ("attention", "train"):
        mask = dict(scale=s["scale"], causal=s["causal"], k_len=s["k_len"], bias=s["bias"])
        o, stat = ctx.fs_attention(s["q"], s["k"], s["v"], **mask)
        out = {"o": o, "stat": stat}
        if s["op"] == "train":
            grads = ctx.fs_attention_grad(s["q"], s["k"], s["v"], o, stat, s["do"], want_bias=s["bias"] is not None, **mask)
            out.update(zip(("dq", "dk", "dv", "dbias"), grads))
        return out
    if s["op"] == "norm":
        y, stat = ctx.fs_layer_norm(s["x"], s["gamma"], s["beta"], s["eps"])
        dx, dgamma, dbeta = ctx.fs_layer_norm_grad(s["x"], s["gamma"], stat, s["dy"])
        return {"y": y, "stat": stat, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    s["adamw"].step(s["grads"])
    return {k: s[k] for k in ("p", "master", "m", "v", "m_scale", "v_scale") if s.get(k) is not None}


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    if case["op"] == "norm":
        e = 4 if case["dtype"] == "f32" else 2
        n = case["rows"] * case["cols"]
        # forward: x read, y written; backward: x and dy read, dx written
        return {"bytes": 5 * e * n + 16 * case["rows"] + 20 * case["cols"], "flops": 20 * n}
    if case["op"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        e = 4 if case["dtype"] == "f32" else 2
        weights = 8 + e if case["master"] else 2 * e
        return {"bytes": n * (weights + e + (16 if case["bits"] == 32 else 4 + 16 / _BLOCK)), "flops": 16 * n}
    e = 4 if case["dtype"] == "f32" else 2
    b, n, m, h, hk, d = (case[k] for k in ("batch", "n", "m", "heads", "kv_heads", "d"))
    pairs, keys = 0, 0
    for length in _lengths(case):
        keys += length
        if case["causal"]:   # row i sees i + length - n + 1 keys
            first = max(0, n - length)
            seen = n - first
            pairs += seen * (first + length - n + 1) + seen * (seen - 1) // 2
        else:
            pairs += n * length
    rows = e * d * h * b * n
    kv = e * d * hk * keys
    if case["op"] == "attention":
        return {"bytes": 2 * rows + 2 * kv + 8 * h * b * n, "flops": 4 * pairs * h * d}
    # (backward: q, o, do and the statistics, k and v read; dq, dk and dv written)
    return {"bytes": 6 * rows + 6 * kv + 16 * h * b * n, "flops": 14 * pairs * h * d}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _exact_attention(case, seed):
    s = _attention_inputs(case, seed)
    b, n, m, h, hk, d = (case[k] for k in ("batch", "n", "m", "heads", "kv_heads", "d"))
    train, group, dev = case["op"] == "train", h // hk, "cuda:0"
    f8 = dict(dtype=torch.float64, device=dev)
    out = {"o": torch.zeros(b, n, h, d, **f8), "stat": torch.zeros(b, h, n, 2, **f8)}
    if train:
        out.update(dq=torch.zeros(b, n, h, d, **f8), dk=torch.zeros(b, m, hk, d, **f8), dv=torch.zeros(b, m, hk, d, **f8))
        dbias = torch.zeros(b, m, **f8)
    out["stat"][..., 0] = -math.inf
    chunk = max(1, 200_000_000 // m)
    for i, length in enumerate(_lengths(case)):
        for j in range(h):
            K, V = s["k"][i, :length, j // group].double(), s["v"][i, :length, j // group].double()
            for r0 in range(0, n, chunk):
                Q = s["q"][i, r0:r0 + chunk, j].double()
                S = torch.mm(Q, K.t().contiguous()) * s["scale"]
                if s["bias"] is not None:
                    S = S + s["bias"][i, :length].double()
                if case["causal"]:
                    seen = torch.arange(length, device=dev)[None, :] - torch.arange(r0, r0 + len(Q), device=dev)[:, None] <= length - n
                    S = torch.where(seen, S, torch.full_like(S, -math.inf))
                lse = torch.logsumexp(S, 1)
                big = S.max(1).values
                P = torch.exp(S - torch.where(lse > -math.inf, lse, torch.zeros_like(lse))[:, None])
                O = torch.mm(P, V)
                out["o"][i, r0:r0 + chunk, j] = O
                out["stat"][i, j, r0:r0 + chunk, 0] = big
                out["stat"][i, j, r0:r0 + chunk, 1] = torch.where(lse > -math.inf, torch.exp(lse - big), torch.zeros_like(lse))
                if train:
                    G = s["do"][i, r0:r0 + chunk, j].double()
                    out["dv"][i, :length, j // group] += torch.mm(P.t().contiguous(), G)
                    dS = P * (torch.mm(G, V.t().contiguous()) - (G * O).sum(1, keepdim=True))
                    out["dq"][i, r0:r0 + chunk, j] = torch.mm(dS, K) * s["scale"]
                    out["dk"][i, :length, j // group] += torch.mm(dS.t().contiguous(), Q) * s["scale"]
                    dbias[i, :length] += dS.sum(0)
    if train and case["bias"]:
        out["dbias"] = dbias
    return out


def _exact_norm(case, seed):
    s = _norm_inputs(case, seed)
    x, dy, gamma, beta = (s[k].double() for k in ("x", "dy", "gamma", "beta"))
    var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
    rstd = (var + s["eps"]).rsqrt()
    xh = (x - mean) * rstd
    c = x.shape[1]
    w = gamma * dy
    dx = (c * w - w.sum(1, keepdim=True) - xh * (w * xh).sum(1, keepdim=True)) * rstd / c
    return {"y": torch.addcmul(beta, xh, gamma), "stat": torch.stack([mean[:, 0], rstd[:, 0]], 1), "dx": dx, "dgamma": (dy * xh).sum(0),
            "dbeta": dy.sum(0)}


def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    (b1, b2), t = s["betas"], s["step"] + 1
    p = (s["master"] if case["master"] else s["p"]).double()
    g = s["grad"].double()
    if case["bits"] == 8:
        m = s["m"].double() * s["m_scale"].double().repeat_interleave(_BLOCK)
        v = (s["v"].double() * s["v_scale"].double().repeat_interleave(_BLOCK)) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m += (1 - b1) * (g - m)
    v += (1 - b2) * (g * g - v)
    step = (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + s["eps"])
    p = p - s["lr"] * (step + s["weight_decay"] * p)
    out = {"p": p, "m": m, "v": v}
    if case["master"]:
        out["master"] = p
    if case["bits"] == 8:   # what is kept goes by the rounding of the 32-bit values, dither and all: there is no such value in 64 bits
        out.update(m=None, v=None, m_scale=None, v_scale=None)
    return out


def exact(case, seed):
    return {"attention": _exact_attention, "train": _exact_attention, "norm": _exact_norm, "adamw": _exact_adamw}[case["op"]](case, seed)
