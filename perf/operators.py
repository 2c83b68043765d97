"""The language-model operators around the adaptation pass, as cases to measure.

Three operators that a user of the adapters needs next to fitting them:

* the head loss: softmax cross entropy of hidden states against the vocabulary head, without the
  logits in memory, with the label-column error of the adaptation pass and with its gradients
  (``dH = W^T eps`` is the d-wide top error of the one-shot calibration);
* the adapter projection: ``Y = X W^T + s_a (X A_a) B_a^T`` for tokens of many requests, each with
  its own adapter ``a`` (or none), and the gradients for ``X``, ``A`` and ``B``;
* the global norm of many gradient tensors, and their clipping.

``run`` computes them in plain torch operations (``own = False``) or through this repository's
library (``own = True``).  Sizes are those of the synthetic workloads: widths 896, 2048, 3584 and
5120, vocabularies of 49152 and 151936, adapter ranks 8 to 32.
"""

import math

import torch

own = False


def listed():
    return [
        # scoring a handful of answer tokens against the label words: latency, the head is read once
        dict(name="head_score", op="head", n=37, d=2048, v=49152, c=4, masked=0.0, weights=False, dh=False, dw=False),
        # the head error of one adaptation pass from the hidden states: most positions are prompt
        dict(name="head_error", op="head", n=16384, d=2048, v=49152, c=4, masked=0.5, weights=False, dh=False, dw=False),
        # probe backward of the calibration: frozen head, the d-wide top error only
        dict(name="head_probe", op="head", n=1531, d=5120, v=151936, c=0, masked=0.0, weights=False, dh=True, dw=False),
        # one training step with a trained head, a quarter of the positions masked, weighted tokens
        dict(name="head_train", op="head", n=4096, d=2048, v=49152, c=0, masked=0.25, weights=True, dh=True, dw=True),
        # a ragged small model: odd token count and an odd vocabulary
        dict(name="head_ragged", op="head", n=777, d=896, v=32003, c=3, masked=0.1, weights=True, dh=True, dw=True),
        # one token of one request through an adapted projection
        dict(name="adapter_token", op="serve", n=1, d=3584, o=3584, k=16, a=4, requests=1, bare=0.0, f32=True),
        # one decoding step of 64 requests, an adapter each, some requests without one
        dict(name="adapter_decode", op="serve", n=64, d=3584, o=3584, k=16, a=96, requests=64, bare=0.1, f32=True),
        # prompts of eight requests of unequal lengths
        dict(name="adapter_prompt", op="serve", n=8192, d=2048, o=2048, k=32, a=8, requests=8, bare=0.1, f32=True),
        # training step of one small adapter: forward, then the gradients
        dict(name="adapter_train", op="train", n=16384, d=896, o=896, k=8, a=1, requests=1, bare=0.0, f32=True),
        # training step of four adapters at once in bfloat16, ragged sequences
        dict(name="adapter_train_many", op="train", n=8191, d=3584, o=3584, k=16, a=4, requests=9, bare=0.1, f32=False),
        # gradients of a small model's adapters: 24 blocks, A and B of each
        dict(name="clip_adapters", op="clip", tensors=48, rows=896, cols=8, head=0, f32=True),
        # a large model's adapters and its head
        dict(name="clip_head", op="clip", tensors=96, rows=5120, cols=32, head=49152 * 2048, f32=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["head", "head", "head", "serve", "serve", "train", "clip"])
    if op == "head":
        d, v = 8 * _log(rng, 64, 640), _log(rng, 1000, 151936)
        dh = rng.random() < 0.6
        n = _log(rng, 1, 16384)
        n = max(1, min(n, int(3.0e11 / (d * v))))
        return dict(op=op, n=n, d=d, v=v, c=rng.choice([0, 2, 4, 11]), masked=rng.choice([0.0, 0.1, 0.5, 0.9]),
                    weights=rng.random() < 0.5, dh=dh, dw=dh and rng.random() < 0.6)
    if op == "clip":
        return dict(op=op, tensors=_log(rng, 1, 300), rows=_log(rng, 64, 5120), cols=rng.randint(1, 33),
                    head=rng.choice([0, _log(rng, 10**5, 10**8)]), f32=rng.random() < 0.5)
    d, o, k = 8 * _log(rng, 64, 640), 8 * _log(rng, 64, 640), rng.choice([4, 8, 12, 16, 24, 32, 64])
    n = _log(rng, 1 if op == "serve" else 64, 8192)
    requests = min(n, _log(rng, 1, 64))
    return dict(op=op, n=n, d=d, o=o, k=k, a=_log(rng, 1, 96 if op == "serve" else 8), requests=requests,
                bare=rng.choice([0.0, 0.1, 0.3]), f32=rng.random() < 0.6)


def work(case):
    if case["op"] == "head":
        n, d, v = case["n"], case["d"], case["v"]
        live = max(1, round(n * (1.0 - case["masked"])))  # a masked position needs no product
        products = 1 + int(case["dh"]) + int(case["dw"])
        nbytes = 2 * live * d + 2 * v * d + 12 * n + 4 * n * case["c"] + 2 * n * d * int(case["dh"]) + 2 * v * d * int(case["dw"])
        return {"bytes": nbytes, "flops": 2 * live * d * v * products}
    if case["op"] == "clip":
        size = 4 if case["f32"] else 2
        return {"bytes": 2 * (size * case["tensors"] * case["rows"] * case["cols"] + 2 * case["head"]),
                "flops": 3 * (case["tensors"] * case["rows"] * case["cols"] + case["head"])}
    n, d, o, k, a = case["n"], case["d"], case["o"], case["k"], case["a"]
    used = min(a, case["requests"])
    size = 4 if case["op"] == "train" and case["f32"] else 2
    nbytes = 2 * (n * d + n * o + d * o) + size * used * k * (d + o)
    flops = 2 * n * (d * o + k * (d + o))
    if case["op"] == "train":  # dY in, dX out; the gradients of A and B out; U is needed again
        nbytes += 2 * (n * o + n * d) + size * a * k * (d + o)
        flops += 2 * n * (d * o + 3 * k * (d + o))
    return {"bytes": nbytes, "flops": flops}


def _gen(seed, case):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + sum(int(1000 * x) for x in case.values() if isinstance(x, (int, float))))
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def _head_inputs(case, seed):
    g = _gen(seed, case)
    n, d, v = case["n"], case["d"], case["v"]
    s = {"case": case}
    y = torch.randint(0, v, (n,), generator=g, device="cuda")
    W = _randn(g, v, d, scale=2.0 / math.sqrt(d), dtype=torch.bfloat16)
    # final-norm hidden states that lean towards the next token's row, about half of them strongly
    lean = 2.0 * (torch.rand((n, 1), generator=g, device="cuda") < 0.5).float()
    s["H"] = (_randn(g, n, d) + lean * W[y].float()).to(torch.bfloat16)
    s["W"] = W
    if case["c"]:  # label words, and answers among them for some of the tokens
        cols = torch.randperm(v, generator=g, device="cuda")[: case["c"]]
        s["cols"] = cols.to(torch.int32)
        pick = torch.randint(0, case["c"], (n,), generator=g, device="cuda")
        y = torch.where(torch.rand((n,), generator=g, device="cuda") < 0.5, cols[pick], y)
    drop = torch.rand((n,), generator=g, device="cuda") < case["masked"]
    s["y"] = torch.where(drop, torch.full_like(y, -1), y).to(torch.int32)
    s["w"] = torch.rand((n,), generator=g, device="cuda") + 0.5 if case["weights"] else None
    return s


def _adapter_inputs(case, seed):
    g = _gen(seed, case)
    n, d, o, k, a = case["n"], case["d"], case["o"], case["k"], case["a"]
    dt = torch.float32 if case["f32"] else torch.bfloat16
    s = {"case": case}
    s["X"] = _randn(g, n, d, dtype=torch.bfloat16)
    s["W"] = _randn(g, o, d, scale=1.0 / math.sqrt(d), dtype=torch.bfloat16)
    s["A"] = _randn(g, a, d, k, scale=1.0 / math.sqrt(d), dtype=dt)
    s["B"] = _randn(g, a, o, k, scale=0.3 / math.sqrt(k), dtype=dt)
    s["scale"] = 0.5 + torch.rand((a,), generator=g, device="cuda")
    # requests in a row, of unequal lengths; each with an adapter of its own where there are enough
    cut = torch.rand((n,), generator=g, device="cuda").argsort()[: case["requests"] - 1] + 1
    request = torch.zeros((n + 1,), device="cuda").scatter_(0, cut, 1.0)[:n].cumsum(0).long()
    if a >= case["requests"]:
        of = torch.randperm(a, generator=g, device="cuda")[: case["requests"]]
    else:
        of = torch.randint(0, a, (case["requests"],), generator=g, device="cuda")
    bare = torch.rand((case["requests"],), generator=g, device="cuda") < case["bare"]
    s["ids"] = torch.where(bare, torch.full_like(of, -1), of)[request].to(torch.int32)
    if case["op"] == "train":
        s["dY"] = _randn(g, n, o, scale=0.01, dtype=torch.bfloat16)
    return s


def _clip_inputs(case, seed):
    g = _gen(seed, case)
    dt = torch.float32 if case["f32"] else torch.bfloat16
    grads = [_randn(g, case["rows"], case["cols"], scale=0.01, dtype=dt) for _ in range(case["tensors"])]
    if case["head"]:
        grads.append(_randn(g, case["head"], scale=0.001, dtype=torch.bfloat16))
    return {"case": case, "grads": grads, "max_norm": 1.0}


def prepare(case, seed):
    if case["op"] == "head":
        s = _head_inputs(case, seed)
        n, d, v = case["n"], case["d"], case["v"]
        s["loss"] = torch.empty((n,), device="cuda")
        s["lse"] = torch.empty((n,), device="cuda")
        s["E"] = torch.empty((n, case["c"]), device="cuda") if case["c"] else None
        s["dH"] = torch.empty((n, d), dtype=torch.bfloat16, device="cuda") if case["dh"] else None
        s["dW"] = torch.empty((v, d), dtype=torch.bfloat16, device="cuda") if case["dw"] else None
        if own:  # the scratch memory that a program keeps
            from paper_2608_03020_gb300 import loca

            nbytes = loca.head_loss_workspace_size(n, v, d, case["c"])
            if case["dh"]:
                nbytes = max(nbytes, loca.head_loss_backward_workspace_size(n, v, d, case["dh"], case["dw"]))
            s["ws"] = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
        return s
    if case["op"] == "clip":
        s = _clip_inputs(case, seed)
        # the clipped gradients stand one after the other, in one buffer for each type
        kinds = [t.dtype for t in s["grads"]]
        s["flat"] = {str(kind): torch.empty((sum(t.numel() for t in s["grads"] if t.dtype == kind),), dtype=kind, device="cuda")
                     for kind in set(kinds)}
        parts = {name: list(flat.split([t.numel() for t in s["grads"] if str(t.dtype) == name])) for name, flat in s["flat"].items()}
        s["out"] = [parts[str(t.dtype)].pop(0).view(t.shape) for t in s["grads"]]
        s["norm"] = torch.empty((1,), device="cuda")
        if own:  # the list of gradient tensors, which stays the same from step to step
            from paper_2608_03020_gb300 import loca

            s["clip"] = loca.GradClip(s["grads"], out=s["out"])
        return s
    s = _adapter_inputs(case, seed)
    n, d, o, k, a = case["n"], case["d"], case["o"], case["k"], case["a"]
    s["Y"] = torch.empty((n, o), dtype=torch.bfloat16, device="cuda")
    if case["op"] == "train":
        s["dX"], s["dA"], s["dB"] = torch.empty_like(s["X"]), torch.empty_like(s["A"]), torch.empty_like(s["B"])
    if own:  # the adapters' device layout, the step's token plan (shared by its projections), scratch memory
        from paper_2608_03020_gb300 import loca

        s["set"] = loca.AdapterSet(a, d, o, k)
        if case["op"] == "serve":
            s["set"].pack(s["A"], s["B"], s["scale"])
        s["plan"] = loca.AdapterPlan(s["ids"], a)
        nbytes = loca.adapter_workspace_size(n, d, o, k, a, backward=case["op"] == "train")
        s["ws"] = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
    return s


def _head_plain(s):
    case, H, W, y, w = s["case"], s["H"], s["W"].float(), s["y"].long(), s["w"]
    live = y >= 0
    H = torch.where(live[:, None], H.float(), 0.0)
    z = H @ W.T
    top = z.amax(1, keepdim=True)
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    weight = live.float() if w is None else torch.where(live, w, 0.0)
    at = torch.where(live, y, 0)
    got = {"loss": weight * (lse - z.gather(1, at[:, None])[:, 0]), "lse": torch.where(live, lse, 0.0)}
    if case["c"]:
        cols = s["cols"].long()
        hit = (y[:, None] == cols[None, :]).float()
        got["E"] = weight[:, None] * (torch.exp(z[:, cols] - lse[:, None]) - hit)
    if case["dh"]:
        del z
        dz = p.div_(total).mul_(weight[:, None])
        dz.scatter_add_(1, at[:, None], -weight[:, None])
        scale = 1.0 / case["n"]
        got["dH"] = (scale * (dz @ W)).to(torch.bfloat16)
        if case["dw"]:
            got["dW"] = (scale * (dz.T @ H)).to(torch.bfloat16)
    return got


def _adapter_plain(s):
    case, ids = s["case"], s["ids"].long()
    n, k, a = case["n"], case["k"], case["a"]
    X, W = s["X"].float(), s["W"].float()
    A = s["A"].float().permute(1, 0, 2).reshape(case["d"], a * k)
    B = (s["B"].float() * s["scale"][:, None, None]).permute(1, 0, 2).reshape(case["o"], a * k)
    mine = (ids[:, None] == torch.arange(a, device="cuda")[None, :]).float().repeat_interleave(k, 1)
    U = (X @ A) * mine
    got = {"Y": (X @ W.T + U @ B.T).to(torch.bfloat16)}
    if case["op"] == "train":
        dY, dt = s["dY"].float(), s["A"].dtype
        T = (dY @ B) * mine
        got["dX"] = (dY @ W + T @ A.T).to(torch.bfloat16)
        got["dA"] = (X.T @ T).reshape(case["d"], a, k).permute(1, 0, 2).contiguous().to(dt)
        dB = (dY.T @ U).reshape(case["o"], a, k).permute(1, 0, 2)
        got["dB"] = (dB * s["scale"][:, None, None]).contiguous().to(dt)
    return got


def _clip_plain(s):
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    _ = [o.copy_(t.float() * factor) for t, o in zip(s["grads"], s["out"])]
    return {"norm": norm.reshape(1), "out": s["flat"]}


def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "head":
            return _head_plain(s)
        if case["op"] == "clip":
            return _clip_plain(s)
        return _adapter_plain(s)
    from paper_2608_03020_gb300 import loca

    if case["op"] == "head":
        loca.loca_head_loss(s["H"], s["W"], s["y"], s["loss"], lse=s["lse"], w=s["w"], label_cols=s.get("cols"),
                            E=s["E"], workspace=s["ws"])
        got = {"loss": s["loss"], "lse": s["lse"]}
        if case["c"]:
            got["E"] = s["E"]
        if case["dh"]:
            loca.loca_head_loss_backward(s["H"], s["W"], s["y"], s["lse"], dH=s["dH"], dW=s["dW"], w=s["w"],
                                         grad_scale=1.0 / case["n"], workspace=s["ws"])
            got["dH"] = s["dH"]
            if case["dw"]:
                got["dW"] = s["dW"]
        return got
    if case["op"] == "clip":
        s["clip"].run(s["max_norm"], s["norm"])
        return {"norm": s["norm"], "out": s["flat"]}
    if case["op"] == "train":  # the adapters change at every step: laid out within the step
        s["set"].pack(s["A"], s["B"], s["scale"])
    loca.loca_adapter_apply(s["X"], s["W"], s["set"], s["plan"], s["Y"], workspace=s["ws"])
    got = {"Y": s["Y"]}
    if case["op"] == "train":
        loca.loca_adapter_backward(s["X"], s["dY"], s["W"], s["set"], s["plan"], dX=s["dX"], dA=s["dA"], dB=s["dB"],
                                   workspace=s["ws"])
        got.update(dX=s["dX"], dA=s["dA"], dB=s["dB"])
    return got


def _head_exact(case, seed):
    s = _head_inputs(case, seed)
    n, d, c = case["n"], case["d"], case["c"]
    W = s["W"].double()
    f64 = dict(dtype=torch.float64, device="cuda")
    got = {"loss": torch.zeros((n,), **f64), "lse": torch.zeros((n,), **f64)}
    if c:
        got["E"] = torch.zeros((n, c), **f64)
    if case["dh"]:
        got["dH"] = torch.zeros((n, d), **f64)
    if case["dw"]:
        got["dW"] = torch.zeros((case["v"], d), **f64)
    live = torch.nonzero(s["y"] >= 0)[:, 0]
    for rows in live.split(2048):
        H, y = s["H"][rows].double(), s["y"][rows].long()
        w = torch.ones((len(rows),), **f64) if s["w"] is None else s["w"][rows].double()
        logp = torch.log_softmax(H @ W.T, 1)
        at = torch.arange(len(rows), device="cuda")
        got["loss"][rows] = -w * logp[at, y]
        # log p of the target is its logit minus the normaliser
        got["lse"][rows] = (H * W[y]).sum(1) - logp[at, y]
        error = logp.exp_()
        error[at, y] -= 1.0
        error *= w[:, None]
        if c:
            got["E"][rows] = error[:, s["cols"].long()]
        if case["dh"]:
            got["dH"][rows] = error @ W / n
        if case["dw"]:
            got["dW"] += error.T @ H / n
    return got


def _adapter_exact(case, seed):
    s = _adapter_inputs(case, seed)
    X, W = s["X"].double(), s["W"].double()
    train = case["op"] == "train"
    got = {"Y": X @ W.T}
    if train:
        dY = s["dY"].double()
        got["dX"], got["dA"], got["dB"] = dY @ W, torch.zeros_like(s["A"]).double(), torch.zeros_like(s["B"]).double()
    for a in range(case["a"]):
        rows = torch.nonzero(s["ids"] == a)[:, 0]
        A, B, scale = s["A"][a].double(), s["B"][a].double(), s["scale"][a].double()
        U = X[rows] @ A
        got["Y"][rows] += scale * (U @ B.T)
        if train:
            T = scale * (dY[rows] @ B)
            got["dX"][rows] += T @ A.T
            got["dA"][a] = X[rows].T @ T
            got["dB"][a] = scale * (dY[rows].T @ U)
    return got


def exact(case, seed):
    if case["op"] == "head":
        return _head_exact(case, seed)
    if case["op"] == "serve" or case["op"] == "train":
        return _adapter_exact(case, seed)
    s = _clip_inputs(case, seed)
    grads = [t.double() for t in s["grads"]]
    norm = math.sqrt(math.fsum(float((t * t).sum()) for t in grads))
    factor = min(1.0, s["max_norm"] / norm) if norm > 0 else 1.0
    kinds = {str(t.dtype) for t in s["grads"]}
    return {"norm": torch.full((1,), norm, dtype=torch.float64, device="cuda"),
            "out": {kind: torch.cat([factor * g.reshape(-1) for g, t in zip(grads, s["grads"]) if str(t.dtype) == kind]) for kind in kinds}}
