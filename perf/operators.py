"""The two ends of a training step around the convolutions, as cases that can be timed and compared.

  "loss"  softmax cross entropy of a linear classifier over many classes, whose logits are never kept: the loss of
          every row and its gradients ("both"), or the loss alone as an evaluation pass has it ("fwd")
  "orth"  the orthogonalised form of a batch of weight gradients (Newton-Schulz products)
  "muon"  the optimiser's whole step: momentum, orthogonalisation, weight decay and update, in place

Sizes: filters of ResNet-18/50 as [K, C*R*S] matrices and their classifiers, and generic ones for large class sets
and large weight matrices.  Where `own` is false the operators run in elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# the quintic of the Newton-Schulz step, and what keeps a gradient of zeros from dividing by zero
COEF, EPS = (3.4445, -4.7750, 2.0315), 1e-7
STEPS, MOMENTUM, KEEP, LR = 5, 0.95, 0.9998, 0.02
IGNORE = -100


def _loss(name, T, D, V, dtype="bf16", bias=1, out=0.0, do="both"):
    return dict(name=name, op="loss", do=do, T=T, D=D, V=V, dtype=dtype, bias=bias, out=out)


def _mat(name, op, B, m, n, dtype):
    return dict(name=name, op=op, B=B, m=m, n=n, dtype=dtype)


def listed():
    return [
        # a single image or token against the 1000 classes of ImageNet: launches and latency are all there is
        _loss("loss 1x512 1000", 1, 512, 1000),
        # the classifier of ResNet-50 under training with 64 images, in single precision
        _loss("loss 64x2048 1000 f32", 64, 2048, 1000, dtype="f32"),
        # a classifier over 21841 classes, an odd number, with a batch as large as the framework's benchmark has
        _loss("loss 256x512 21841", 256, 512, 21841),
        # odd everything, a third of the rows left out, no bias: sequences with padding and masked prompts
        _loss("loss 1531x1001 50257 f32", 1531, 1001, 50257, dtype="f32", bias=0, out=0.35),
        # evaluation over a middling class set
        _loss("eval 4096x1024 32000", 4096, 1024, 32000, bias=0, do="fwd"),
        # the largest: logits that would take 4.3 GB in 32 bits
        _loss("loss 8192x4096 131072", 8192, 4096, 131072, bias=0, out=0.1),
        # one 1x1 filter of the first stage of ResNet-50: latency
        _mat("orth 64x64", "orth", 1, 64, 64, "f32"),
        # the four 3x3 filters of ResNet-18's first stage in one call
        _mat("muon 4 of 64x576", "muon", 4, 64, 576, "bf16"),
        # the last stage's three, each with 2.4 million weights
        _mat("orth 3 of 512x4608", "orth", 3, 512, 4608, "f32"),
        # the expansions of ResNet-50's last stage: more rows than columns
        _mat("muon 3 of 2048x512", "muon", 3, 2048, 512, "f32"),
        # a classifier's weights: nothing divides the tile
        _mat("orth 1000x2049 bf16", "orth", 1, 1000, 2049, "bf16"),
        # the largest: a square weight matrix of a wide layer
        _mat("muon 4096x4096", "muon", 1, 4096, 4096, "bf16"),
    ]


MAX_LOSS, MAX_LOGITS, MAX_MAT = 8192 * 4096 * 131072, 8192 * 131072, 4 * 4096.0 ** 3


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A size between lo and hi, as it comes or (more often) a multiple of 8; never 3072."""
    n = _log_int(rng, lo, hi)
    n = n if rng.random() < 0.4 else max(8, (n + 4) // 8 * 8)
    return n + 8 if n == 3072 else n


def draw(rng):
    if rng.random() < 0.5:
        c = dict(op="loss", do=rng.choice(["both", "both", "both", "fwd"]), T=_extent(rng, 1, 16384), D=_extent(rng, 64, 4096),
                 V=_extent(rng, 10, 131072), dtype=rng.choice(["bf16", "bf16", "f32"]), bias=rng.choice([0, 1]),
                 out=rng.choice([0.0, 0.0, 0.1, 0.5]))
        cap = MAX_LOSS // (8 if c["dtype"] == "f32" else 1)
        while c["T"] * c["D"] * c["V"] > cap or c["T"] * c["V"] > MAX_LOGITS:
            c["V" if c["V"] >= c["T"] else "T"] = max(c["V"], c["T"]) // 2
        return c
    c = dict(op=rng.choice(["orth", "muon"]), B=rng.choice([1, 1, 2, 3, 4, 8]), m=_extent(rng, 16, 4096), n=_extent(rng, 16, 8192),
             dtype=rng.choice(["f32", "bf16"]))
    while c["B"] * _products(c) > MAX_MAT:
        if c["B"] > 1:
            c["B"] //= 2
        else:
            c["m" if c["m"] >= c["n"] else "n"] //= 2
    return c


def _products(case):
    """Multiply-adds of one Newton-Schulz step of one matrix, twice: of a symmetric product only half is needed."""
    r, c = sorted((case["m"], case["n"]))
    return 3.0 * r * r * c + 1.0 * r * r * r


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "loss":
        T, D, V = case["T"], case["D"], case["V"]
        live = T * (1 - case["out"])
        n = (live * D + V * D + case["bias"] * V) * e + T * 8 + T * 8
        if case["do"] == "fwd":
            return {"bytes": n, "flops": 2 * live * D * V}
        return {"bytes": n + T * 4 + (T * D + V * D) * e + case["bias"] * V * e, "flops": 6 * live * D * V}
    size = case["B"] * case["m"] * case["n"]
    # the gradient in; the result out, or momentum and weights in and out
    moved = size * (4 + e if case["op"] == "orth" else 4 + 8 + 2 * e)
    return {"bytes": moved, "flops": STEPS * case["B"] * _products(case)}


def _inputs(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    td = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEV).mul_(std)

    if case["op"] == "loss":
        T, D, V = case["T"], case["D"], case["V"]
        # features after a normalisation, weights that make logits of a spread of about 2, a mean over the rows as loss
        t = {"H": normal(T, D).to(td), "W": normal(V, D, std=2 / math.sqrt(D)).to(td)}
        t["labels"] = torch.randint(0, V, (T,), generator=g, device=DEV)
        t["labels"].masked_fill_(torch.rand(T, generator=g, device=DEV) < case["out"], IGNORE)
        t["gloss"] = torch.full((T,), 1.0 / T, device=DEV)
        if case["bias"]:
            t["b"] = normal(V, std=0.5).to(td)
        return t
    B, m, n = case["B"], case["m"], case["n"]
    # a weight gradient: a few strong directions whose strength falls off, over noise
    r = min(m, n, 32)
    fall = torch.exp(-0.15 * torch.arange(r, device=DEV))
    grad = (normal(B, m, r) * fall) @ normal(B, r, n, std=1e-3) + normal(B, m, n, std=2e-4)
    if case["op"] == "orth":
        return {"G": grad}
    return {"G": grad, "M": normal(B, m, n, std=1e-3) + 5 * grad, "W": normal(B, m, n, std=math.sqrt(2.0 / n)).to(td)}


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


def _kept(s):
    """What a program keeps beside its data: descriptor, outputs and workspace."""
    from paper_2409_11902_amd import binding as B
    c = s["case"]

    def scratch(n):
        return torch.empty(max(16, n), dtype=torch.uint8, device=DEV)

    if c["op"] == "loss":
        d = B.make_loss_desc(c["T"], c["D"], c["V"], dtype=B.F32 if c["dtype"] == "f32" else B.BF16, has_bias=c["bias"],
                             ignore_index=IGNORE)
        ops = (B.LOSS_FWD,) if c["do"] == "fwd" else (B.LOSS_FWD, B.LOSS_BWD)
        k = {"B": B, "d": d, "ws": scratch(max(B.cac_loss_workspace_size(d, op) for op in ops)),
             "loss": torch.empty(c["T"], device=DEV), "lse": torch.empty(c["T"], device=DEV)}
        if c["do"] == "both":
            k.update(dH=torch.empty_like(s["H"]), dW=torch.empty_like(s["W"]), db=torch.empty_like(s["b"]) if c["bias"] else None)
    else:
        d = B.make_muon_desc(c["m"], c["n"], batch=c["B"], dtype=B.F32 if c["dtype"] == "f32" else B.BF16, steps=STEPS)
        op = B.MUON_ORTHOGONALISE if c["op"] == "orth" else B.MUON_STEP
        k = {"B": B, "d": d, "ws": scratch(B.cac_muon_workspace_size(d, op))}
        if c["op"] == "orth":
            k["O"] = torch.empty(s["G"].shape, dtype=TYPES[c["dtype"]], device=DEV)
    s["kept"] = k
    return k


def _run_own(s):
    k = s.get("kept") or _kept(s)
    B, d, ws = k["B"], k["d"], k["ws"]
    c = s["case"]
    if c["op"] == "loss":
        B.cac_loss_fwd(d, s["H"], s["W"], s.get("b"), s["labels"], k["loss"], k["lse"], ws)
        if c["do"] == "fwd":
            return {"loss": k["loss"], "lse": k["lse"]}
        B.cac_loss_bwd(d, s["H"], s["W"], s.get("b"), s["labels"], k["lse"], s["gloss"], k["dH"], k["dW"], k["db"], ws)
        r = {"loss": k["loss"], "lse": k["lse"], "dH": k["dH"], "dW": k["dW"]}
        if c["bias"]:
            r["db"] = k["db"]
        return r
    if c["op"] == "orth":
        B.cac_orthogonalise(d, s["G"], k["O"], ws)
        return {"O": k["O"]}
    B.cac_muon_step(d, s["G"], s["M"], s["W"], MOMENTUM, KEEP, LR, ws)
    return {"M": s["M"], "W": s["W"]}


def _orthogonalise(x):
    """Five steps of x <- a x + (b A + c A A) x with A = x x^T, from x over its norm; the shorter side as rows."""
    a, b, c = COEF
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT
    x = x / (x.square().sum(dim=(-2, -1), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.mT if tall else x


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "loss":
        labels = s["labels"]
        live = (labels >= 0) & (labels < c["V"]) & (labels != IGNORE)
        at = torch.where(live, labels, 0).unsqueeze(1)
        h, w = s["H"].float(), s["W"].float()
        z = h @ w.t()
        if c["bias"]:
            z += s["b"].float()
        top = z.amax(dim=1, keepdim=True)
        zy = z.gather(1, at)
        p = z.sub_(top).exp_()
        total = p.sum(dim=1, keepdim=True)
        lse = top + total.log()
        loss = torch.where(live, (lse - zy).squeeze(1), 0.0)
        lse = torch.where(live, lse.squeeze(1), 0.0)
        if c["do"] == "fwd":
            return {"loss": loss, "lse": lse}
        p /= total
        p.scatter_add_(1, at, torch.full_like(zy, -1.0))
        p *= torch.where(live, s["gloss"], 0.0).unsqueeze(1)
        td = s["H"].dtype
        r = {"loss": loss, "lse": lse, "dH": (p @ w).to(td), "dW": (p.t() @ h).to(td)}
        if c["bias"]:
            r["db"] = p.sum(dim=0).to(td)
        return r
    if c["op"] == "orth":
        return {"O": _orthogonalise(s["G"]).to(TYPES[c["dtype"]])}
    s["M"].mul_(MOMENTUM).add_(s["G"])
    step = _orthogonalise(s["G"] + MOMENTUM * s["M"])
    s["W"].copy_(KEEP * s["W"].float() - LR * step)
    return {"M": s["M"], "W": s["W"]}


def exact(case, seed):
    t = {k: v if k == "labels" else v.double() for k, v in _inputs(case, seed).items()}
    if case["op"] == "loss":
        T, V = case["T"], case["V"]
        rows = ((t["labels"] >= 0) & (t["labels"] < V)).nonzero().squeeze(1)  # the rows that count, on their own
        h, y = t["H"][rows], t["labels"][rows]
        z = torch.addmm(t["b"], h, t["W"].t()) if case["bias"] else h @ t["W"].t()
        some = torch.logsumexp(z, dim=1)
        every = torch.arange(len(rows), device=DEV)
        loss, lse = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(2))
        loss[rows], lse[rows] = some - z[every, y], some
        if case["do"] == "fwd":
            return {"loss": loss, "lse": lse}
        z = z.sub_(some.unsqueeze(1)).exp_()
        z[every, y] -= 1
        z *= t["gloss"][rows].unsqueeze(1)
        dh = torch.zeros(T, case["D"], dtype=torch.float64, device=DEV)
        dh[rows] = z @ t["W"]
        r = {"loss": loss, "lse": lse, "dH": dh, "dW": z.t() @ h}
        if case["bias"]:
            r["db"] = z.sum(dim=0)
        return r
    a, b, c = COEF

    def orthogonal(x):
        out = []
        for m in x:  # one matrix at a time, from whichever side is the shorter
            m = m / (torch.linalg.matrix_norm(m) + EPS)
            for _ in range(STEPS):
                wide = m.shape[0] <= m.shape[1]
                s = m @ m.t() if wide else m.t() @ m
                q = a * torch.eye(len(s), dtype=s.dtype, device=DEV) + b * s + c * (s @ s)
                m = q @ m if wide else m @ q
            out.append(m)
        return torch.stack(out)

    if case["op"] == "orth":
        return {"O": orthogonal(t["G"])}
    m = MOMENTUM * t["M"] + t["G"]
    return {"M": m, "W": KEEP * t["W"] - LR * orthogonal(MOMENTUM * m + t["G"])}
