"""The residual block of a training step, as cases that can be timed and compared.

  "linear"  a dense layer, R + alpha * drop(act(X W^T + b)): its forward pass ("fwd") or the gradients of X, W and b
            ("bwd"), which form what act needs once more
  "drop"    dropout with its residual, R + alpha * drop(X), whose mask is a function of a counter and never stored
  "norm"    what stands between two blocks, S = R + alpha * drop(gate * post(F)) and H = pre(S) with norms post and
            pre: forward, or the gradients of R, F, the gate and the norms' weights

Sizes: pooled features and classifiers of ResNet-18/50 (512 and 2048 features), and generic widths.  Where `own` is
false the operators run in elementary torch operations in 32 bits.

The mask (every operator's): Philox 4x32 of ten rounds (Salmon, Moraes, Dror and Shaw, 2011) with key `seed` and counter
(group, site, step), group = row * ceil(columns / 8) + column // 8; a group's eight elements have 16 bits each, from
the low half of the first word on, and those below round(65536 p) are dropped.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu", "silu")
NORMS = ("none", "rms", "layer")
EPS = 1e-5
SITE = 3


def _linear(name, do, T, D, N, dtype="bf16", act="none", bias=1, res=0, p=0.0, alpha=1.0):
    return dict(name=name, op="linear", do=do, T=T, D=D, N=N, dtype=dtype, act=act, bias=bias, res=res, p=p, alpha=alpha)


def _drop(name, T, D, dtype, p, res=0, alpha=1.0):
    return dict(name=name, op="drop", do="fwd", T=T, D=D, dtype=dtype, p=p, res=res, alpha=alpha)


def _norm(name, do, T, D, dtype="bf16", post="none", pre="rms", gate=0, p=0.0, alpha=1.0):
    return dict(name=name, op="norm", do=do, T=T, D=D, dtype=dtype, post=post, pre=pre, gate=gate, p=p, alpha=alpha)


def listed():
    return [
        # the widening layer of a block for a single image or token, as it answers: latency, and reading the weights once
        _linear("linear fwd 1x512 2048 gelu", "fwd", 1, 512, 2048, act="gelu"),
        # answers for a few at a time: the narrowing layer on its residual; the weights' bandwidth
        _linear("linear fwd 16x8192 2048", "fwd", 16, 8192, 2048, res=1),
        # single precision and odd everything, as a batch of ragged lengths laid end to end has it
        _linear("linear bwd 1531x1001 515 f32", "bwd", 1531, 1001, 515, dtype="f32", act="silu"),
        # the widening layer of a block under training: the largest forward pass
        _linear("linear fwd 8192x2048 8192 gelu", "fwd", 8192, 2048, 8192, act="gelu", p=0.1),
        # the gradients of a block's widening layer with dropout behind the activation
        _linear("linear bwd 4096x2048 8192 gelu", "bwd", 4096, 2048, 8192, act="gelu", p=0.1),
        # the gradients of a narrowing layer with dropout before its residual: the largest
        _linear("linear bwd 8192x8192 2048", "bwd", 8192, 8192, 2048, p=0.1, alpha=0.5),
        # dropout on the pooled features of a small batch in front of a classifier: latency
        _drop("drop 64x512 f32", 64, 512, "f32", 0.5),
        # dropout on a block's residual under training: bandwidth
        _drop("drop 16384x4096", 16384, 4096, "bf16", 0.1, res=1),
        # the norm in front of a block for a single token that is being answered: latency
        _norm("norm fwd 1x2048", "fwd", 1, 2048),
        # between two blocks under training, a norm behind the one and one before the other
        _norm("norm fwd 8192x4096", "fwd", 8192, 4096, post="rms", pre="rms", p=0.1, alpha=0.7),
        # gradients in single precision, odd widths, every image (of 7x7 pixels) with a gate of its own
        _norm("norm bwd 3136x1001 f32", "bwd", 3136, 1001, dtype="f32", post="layer", pre="layer", gate=49),
        # gradients between two blocks under training with a learned gate for each feature
        _norm("norm bwd 8192x2048", "bwd", 8192, 2048, post="rms", pre="layer", gate=8192, p=0.1),
    ]


MAX_PRODUCT = 8192 * 8192 * 2048          # multiply-adds of one product
MAX_ELEMENTS = 16384 * 4096


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A size between lo and hi, as it comes or (more often) a multiple of 8."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.4 else max(8, (n + 4) // 8 * 8)


def draw(rng):
    op = rng.choice(["linear", "linear", "drop", "norm", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    p = rng.choice([0.0, 0.0, 0.1, 0.1, 0.5, 0.25])
    alpha = rng.choice([1.0, 1.0, 0.5, -0.3])
    if op == "linear":
        c = dict(op=op, do=rng.choice(["fwd", "bwd"]), T=_extent(rng, 1, 16384), D=_extent(rng, 16, 8192), N=_extent(rng, 16, 8192),
                 dtype=dtype, act=rng.choice(ACTS), bias=rng.choice([0, 1, 1]), res=rng.choice([0, 1]), p=p, alpha=alpha)
        # (no dearer than the largest listed case: three products with an activation's gradient, and float's rate)
        cap = MAX_PRODUCT // (16 if dtype == "f32" else 2)
        while c["T"] * c["D"] * c["N"] > cap:
            k = max(("T", "D", "N"), key=lambda k: c[k])
            c[k] //= 2
        return c
    if op == "drop":
        c = dict(op=op, do="fwd", T=_extent(rng, 1, 65536), D=_extent(rng, 1, 16384), dtype=dtype, p=p or 0.1, res=rng.choice([0, 1]), alpha=alpha)
    else:
        c = dict(op=op, do=rng.choice(["fwd", "bwd"]), T=_extent(rng, 1, 65536), D=_extent(rng, 16, 16384), dtype=dtype,
                 post=rng.choice(NORMS), pre=rng.choice(NORMS), gate=0, p=p, alpha=alpha)
    while c["T"] * c["D"] > MAX_ELEMENTS // 2:
        c["T" if c["T"] >= c["D"] else "D"] //= 2
    if op == "norm" and rng.random() < 0.5:
        c["gate"] = c["T"] if rng.random() < 0.5 else _log_int(rng, 1, c["T"])
    return c


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    T, D = case["T"], case["D"]
    if case["op"] == "linear":
        N = case["N"]
        n = (T * D + N * D + case["bias"] * N) * e
        if case["do"] == "fwd":
            return {"bytes": n + (1 + case["res"]) * T * N * e, "flops": 2 * T * D * N}
        return {"bytes": 2 * n + T * N * e, "flops": (6 if case["act"] != "none" else 4) * T * D * N}
    if case["op"] == "drop":
        return {"bytes": (2 + case["res"]) * T * D * e, "flops": 3 * T * D}
    post, pre, gate = case["post"] != "none", case["pre"] != "none", case["gate"] > 0
    gates = -(-T // case["gate"]) * D if gate else 0
    params = 4 * (D * (NORMS.index(case["post"]) + NORMS.index(case["pre"])) + gates)
    if case["do"] == "fwd":
        return {"bytes": (3 + pre) * T * D * e + params, "flops": (4 + 6 * post + 6 * pre) * T * D}
    # F is needed where there is a norm behind the block or a gate, S where there is one in front of the next
    return {"bytes": ((post or gate) + pre * 2 + 3) * T * D * e + 2 * params, "flops": (6 + 12 * post + 12 * pre) * T * D}


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    td = TYPES[case["dtype"]]
    T, D = case["T"], case["D"]

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device=DEV).mul_(std).add_(mean)

    t = {"rng": torch.randint(0, 1 << 62, (2,), generator=g, device=DEV)}
    if case["op"] == "linear":
        N = case["N"]
        # features behind a norm, weights that make pre-activations of a spread of about 1, gradients of a mean over the rows
        t["X"], t["W"] = normal(T, D).to(td), normal(N, D, std=1 / math.sqrt(D)).to(td)
        if case["bias"]:
            t["b"] = normal(N, std=0.2).to(td)
        if case["do"] == "bwd":
            t["dY"] = normal(T, N, std=1.0 / T).to(td)
        elif case["res"]:
            t["R"] = normal(T, N, std=2.0).to(td)
        return t
    if case["op"] == "drop":
        t["X"] = normal(T, D).to(td)
        if case["res"]:
            t["R"] = normal(T, D, std=2.0).to(td)
        return t
    # rows of different scale, a few features that are large in all of them
    wide = normal(D).abs_().mul_(0.5).add_(0.5)
    wide[torch.randint(0, D, (max(1, D // 256),), generator=g, device=DEV)] *= 10
    rows = torch.rand(T, 1, generator=g, device=DEV).add_(0.5)
    t["F"] = (normal(T, D, mean=0.1) * rows * wide).to(td)
    if case["do"] == "fwd":
        t["R"] = (normal(T, D, std=1.5) * wide).to(td)
    else:
        t["S"] = (normal(T, D, std=1.5, mean=-0.05) * wide).to(td)
        t["dS"] = normal(T, D, std=1.0 / T).to(td)
        if case["pre"] != "none":
            t["dH"] = normal(T, D, std=1.0 / T).to(td)
    if case["gate"]:
        t["gate"] = normal(-(-T // case["gate"]), D, std=0.3, mean=0.5)
    for k in ("post", "pre"):
        if case[k] != "none":
            t["w_" + k] = normal(D, std=0.1, mean=1.0)
        if case[k] == "layer":
            t["b_" + k] = normal(D, std=0.1)
    return t


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


# ---- the framework's calls

def _kept(s):
    """What a program keeps beside its data: descriptor, outputs and workspace."""
    from paper_2409_11902_amd import binding as B
    c = s["case"]
    T, D, td = c["T"], c["D"], TYPES[c["dtype"]]
    common = dict(dtype=B.F32 if c["dtype"] == "f32" else B.BF16, alpha=c["alpha"], p=c["p"], site=SITE)

    def new(*shape, dtype=td):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    k = {"B": B, "rng": s["rng"] if c["p"] > 0 else None}
    need = 0
    if c["op"] == "linear":
        d = B.make_linear_desc(T, D, c["N"], act=ACTS.index(c["act"]), has_bias=c["bias"], **common)
        need = B.cac_linear_workspace_size(d, B.LINEAR_FWD if c["do"] == "fwd" else B.LINEAR_BWD)
        if c["do"] == "fwd":
            k["Y"] = new(T, c["N"])
        else:
            k.update(dX=new(T, D), dW=new(c["N"], D), db=new(c["N"]) if c["bias"] else None)
    elif c["op"] == "drop":
        d = B.make_dropout_desc(T, D, **common)
        k["Y"] = new(T, D)
    else:
        d = B.make_block_norm_desc(T, D, post=NORMS.index(c["post"]), pre=NORMS.index(c["pre"]), gate_rows=c["gate"], eps_post=EPS, eps_pre=EPS,
                                   **common)
        need = B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_FWD if c["do"] == "fwd" else B.BLOCK_NORM_BWD)
        if c["do"] == "fwd":
            k.update(S=new(T, D), H=new(T, D) if c["pre"] != "none" else None)
        else:
            k.update(dR=new(T, D), dF=new(T, D))
            for name in ("gate", "w_post", "b_post", "w_pre", "b_pre"):
                k["d" + name] = torch.empty_like(s[name]) if name in s else None
    k.update(d=d, ws=new(max(16, need), dtype=torch.uint8))
    s["kept"] = k
    return k


def _run_own(s):
    k = s.get("kept") or _kept(s)
    B, d, ws, c = k["B"], k["d"], k["ws"], s["case"]
    if c["op"] == "linear":
        if c["do"] == "fwd":
            B.cac_linear_fwd(d, s["X"], s["W"], s.get("b"), s.get("R"), k["rng"], k["Y"], ws)
            return {"Y": k["Y"]}
        B.cac_linear_bwd(d, s["X"], s["W"], s.get("b"), s["dY"], k["rng"], k["dX"], k["dW"], k["db"], ws)
        names = ("dX", "dW", "db")
    elif c["op"] == "drop":
        B.cac_dropout(d, s["X"], s.get("R"), k["rng"], k["Y"])
        return {"Y": k["Y"]}
    elif c["do"] == "fwd":
        B.cac_block_norm_fwd(d, s["F"], s["R"], s.get("gate"), s.get("w_post"), s.get("b_post"), s.get("w_pre"), s.get("b_pre"), k["rng"],
                             k["S"], k["H"])
        names = ("S", "H")
    else:
        B.cac_block_norm_bwd(d, s["F"], s["S"], s.get("gate"), s.get("w_post"), s.get("b_post"), s.get("w_pre"), s.get("dH"), s["dS"], k["rng"],
                             k["dR"], k["dF"], k["dgate"], k["dw_post"], k["db_post"], k["dw_pre"], k["db_pre"], ws)
        names = ("dR", "dF", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")
    return {n: k[n] for n in names if k[n] is not None}


# ---- the plain form

LOW = 0xFFFFFFFF


def _random16(rng, rows, cols):
    """16 random bits for every element, [rows][cols]: words in 64 bits, so that a product of two of them is whole."""
    seed, step = rng[0], rng[1]
    wide = -(-cols // 8)
    g = torch.arange(rows * wide, device=rng.device)
    c = [g & LOW, (g >> 32) | (SITE << 8), (step & LOW).expand_as(g), ((step >> 32) & LOW).expand_as(g)]
    k0, k1 = seed & LOW, (seed >> 32) & LOW
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((b >> 32) & LOW) ^ c[1] ^ k0, b & LOW, ((a >> 32) & LOW) ^ c[3] ^ k1, a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    r = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], dim=1)
    return r.view(rows, wide * 8)[:, :cols]


def _threshold(p):
    return int(p * 65536 + 0.5)


def _dropped(c, rng, x, cols):
    """alpha * drop(x) in 32 bits."""
    if c["p"] == 0:
        return x * c["alpha"]
    t = _threshold(c["p"])
    return torch.where(_random16(rng, c["T"], cols) >= t, x * (c["alpha"] * (65536.0 / (65536 - t))), 0.0)


def _activation(act, u):
    """act(u) and its derivative."""
    if act == "relu":
        return u.clamp(min=0), (u > 0).to(u.dtype)
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(u * -math.sqrt(0.5))
        return u * phi, phi + u * torch.exp(-0.5 * u * u) * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        s = 1 / (1 + torch.exp(-u))
        return u * s, s * (1 + u * (1 - s))
    return u, torch.ones_like(u)


def _normalised(kind, x):
    """x as the norm leaves it before weights, and one over the spread."""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    inv = 1 / torch.sqrt(x.square().mean(dim=1, keepdim=True) + EPS)
    return x * inv, inv


def _norm_gradient(kind, xhat, inv, g):
    """Gradient of a norm's input from that of xhat."""
    if kind == "none":
        return g
    g = g - xhat * (g * xhat).mean(dim=1, keepdim=True)
    if kind == "layer":
        g = g - g.mean(dim=1, keepdim=True)
    return g * inv


def _affine(s, which, x):
    if "w_" + which in s:
        x = x * s["w_" + which]
    if "b_" + which in s:
        x = x + s["b_" + which]
    return x


def _gate_rows(s):
    c = s["case"]
    return s["gate"].repeat_interleave(c["gate"], dim=0)[:c["T"]]


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    td = TYPES[c["dtype"]]
    if c["op"] == "linear":
        x, w = s["X"].float(), s["W"].float()
        if c["do"] == "fwd" or c["act"] != "none":
            u = x @ w.t()
            if c["bias"]:
                u = u + s["b"].float()
            y, slope = _activation(c["act"], u)
        if c["do"] == "fwd":
            y = _dropped(c, s["rng"], y, c["N"])
            if c["res"]:
                y = y + s["R"].float()
            return {"Y": y.to(td)}
        g = _dropped(c, s["rng"], s["dY"].float(), c["N"])
        if c["act"] != "none":
            g = g * slope
        r = {"dX": (g @ w).to(td), "dW": (g.t() @ x).to(td)}
        if c["bias"]:
            r["db"] = g.sum(dim=0).to(td)
        return r
    if c["op"] == "drop":
        y = _dropped(c, s["rng"], s["X"].float(), c["D"])
        return {"Y": (y + s["R"].float() if c["res"] else y).to(td)}
    f = s["F"].float()
    fhat, finv = _normalised(c["post"], f)
    n = _affine(s, "post", fhat)
    gate = _gate_rows(s) if c["gate"] else None
    if c["do"] == "fwd":
        total = s["R"].float() + _dropped(c, s["rng"], n * gate if c["gate"] else n, c["D"])
        r = {"S": total.to(td)}
        if c["pre"] != "none":
            r["H"] = _affine(s, "pre", _normalised(c["pre"], total)[0]).to(td)
        return r
    total = s["dS"].float()
    sums = {}
    if c["pre"] != "none":
        shat, sinv = _normalised(c["pre"], s["S"].float())
        dh = s["dH"].float()
        total = total + _norm_gradient(c["pre"], shat, sinv, dh * s["w_pre"])
        sums["w_pre"], sums["b_pre"] = dh * shat, dh
    a = _dropped(c, s["rng"], total, c["D"])
    dn = a
    if c["gate"]:
        whole = torch.zeros(s["gate"].shape[0] * c["gate"], c["D"], device=DEV)
        whole[:c["T"]] = a * n
        dgate = whole.view(-1, c["gate"], c["D"]).sum(dim=1)
        dn = a * gate
    sums["w_post"], sums["b_post"] = dn * fhat, dn
    r = {"dR": total.to(td)}
    r["dF"] = _norm_gradient(c["post"], fhat, finv, dn * s["w_post"] if "w_post" in s else dn).to(td)
    if c["gate"]:
        r["dgate"] = dgate
    for name in ("w_post", "b_post", "w_pre", "b_pre"):
        if name in s:
            r["d" + name] = sums[name].sum(dim=0)
    return r


# ---- the definition in 64 bits

def _times(a, m):
    """High and low word of a * m, the sixteen-bit halves multiplied apart."""
    a0, a1, m0, m1 = a % 65536, a // 65536, m % 65536, m // 65536
    low, mid = a0 * m0, a0 * m1 + a1 * m0
    low = low + (mid % 65536) * 65536
    return a1 * m1 + mid // 65536 + low // (1 << 32), low % (1 << 32)


def _keeps(case, rng, cols):
    """1 / (1 - p) where an element is kept, else 0."""
    T, p = case["T"], case["p"]
    if p == 0:
        return 1.0
    seed, step = (int(v) for v in rng.cpu())
    across = (cols + 7) // 8
    row = torch.arange(T, device=DEV).unsqueeze(1)
    group = (row * across + torch.arange(across, device=DEV)).flatten()
    x0, x1 = group % (1 << 32), group // (1 << 32) + SITE * 256
    x2, x3 = torch.full_like(group, step % (1 << 32)), torch.full_like(group, step // (1 << 32))
    for turn in range(10):
        key0 = (seed + turn * 0x9E3779B9) % (1 << 32)
        key1 = (seed // (1 << 32) + turn * 0xBB67AE85) % (1 << 32)
        h0, l0 = _times(x0, 0xD2511F53)
        h1, l1 = _times(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ key0, l1, h0 ^ x3 ^ key1, l0
    bits = torch.empty(len(group), 8, dtype=torch.int64, device=DEV)
    for i, word in enumerate((x0, x1, x2, x3)):
        bits[:, 2 * i], bits[:, 2 * i + 1] = word % 65536, word // 65536
    limit = math.floor(p * 65536 + 0.5)
    return (bits.view(T, across * 8)[:, :cols] >= limit).double() / (1 - limit / 65536)


def _exact_linear(case, t):
    u = t["X"] @ t["W"].t() + t.get("b", 0.0)
    keep = _keeps(case, t["rng"], case["N"]) * case["alpha"]
    act = case["act"]
    if act == "gelu":
        cdf = torch.special.ndtr(u)
        y, slope = u * cdf, cdf + u * torch.exp(u.square() / -2) / math.sqrt(2 * math.pi)
    elif act == "silu":
        y = u * torch.sigmoid(u)
        slope = torch.sigmoid(u) + y * torch.sigmoid(-u)
    elif act == "relu":
        y, slope = torch.where(u > 0, u, 0.0), torch.where(u > 0, 1.0, 0.0)
    else:
        y, slope = u, 1.0
    if case["do"] == "fwd":
        return {"Y": t.get("R", 0.0) + keep * y}
    g = t["dY"] * keep * slope
    r = {"dX": g @ t["W"], "dW": g.t() @ t["X"]}
    if case["bias"]:
        r["db"] = g.sum(dim=0)
    return r


def _exact_norm(case, t):
    T, D = case["T"], case["D"]

    def statistics(kind, x):
        centre = x.mean(dim=1, keepdim=True) if kind == "layer" else 0.0
        return centre, (((x - centre) ** 2).sum(dim=1, keepdim=True) / D + EPS).rsqrt()

    def through(kind, x, weight, bias):
        if kind == "none":
            return x
        centre, inv = statistics(kind, x)
        return (x - centre) * inv * weight + (0.0 if bias is None else bias)

    def back(kind, x, weight, g):
        """Gradients of x and of the weights."""
        centre, inv = statistics(kind, x)
        y, gw = (x - centre) * inv, g * weight
        dx = gw - y * (gw * y).sum(dim=1, keepdim=True) / D
        if kind == "layer":
            dx = dx - gw.sum(dim=1, keepdim=True) / D
        return dx * inv, (g * y).sum(dim=0)

    keep = _keeps(case, t["rng"], D) * case["alpha"]
    group = torch.arange(T, device=DEV) // case["gate"] if case["gate"] else None
    gate = t["gate"][group] if case["gate"] else 1.0
    n = through(case["post"], t["F"], t.get("w_post"), t.get("b_post"))
    if case["do"] == "fwd":
        s = t["R"] + keep * gate * n
        r = {"S": s}
        if case["pre"] != "none":
            r["H"] = through(case["pre"], s, t["w_pre"], t.get("b_pre"))
        return r
    r = {"dR": t["dS"]}
    if case["pre"] != "none":
        ds, dw = back(case["pre"], t["S"], t["w_pre"], t["dH"])
        r["dR"] = t["dS"] + ds
    g = keep * r["dR"]
    dn = g * gate
    r["dF"] = dn
    if case["post"] != "none":
        r["dF"], dw_post = back(case["post"], t["F"], t["w_post"], dn)
    if case["gate"]:
        r["dgate"] = torch.zeros_like(t["gate"]).index_add_(0, group, g * n)
    if "w_post" in t:
        r["dw_post"] = dw_post
    if "b_post" in t:
        r["db_post"] = dn.sum(dim=0)
    if "w_pre" in t:
        r["dw_pre"] = dw
    if "b_pre" in t:
        r["db_pre"] = t["dH"].sum(dim=0)
    return r


def exact(case, seed):
    t = {k: v if k == "rng" else v.double() for k, v in _inputs(case, seed).items()}
    if case["op"] == "linear":
        return _exact_linear(case, t)
    if case["op"] == "drop":
        y = t["X"] * _keeps(case, t["rng"], case["D"]) * case["alpha"]
        return {"Y": y + t["R"] if case["res"] else y}
    return _exact_norm(case, t)
