"""Operators of the adapted model's blocks, head and served weights, as cases to measure.

* distillation from a teacher's top logits: the student's hidden states against the vocabulary head,
  ``loss = w tau^2 sum_k q_k (log q_k - log p_k)`` with ``q = softmax(t / tau)`` over a position's K
  teacher logits and ``p = softmax(z / tau)`` over the whole vocabulary, without the logits in memory,
  and the gradients of the hidden states and the head;
* the gated feed-forward of a block: ``H = act(X Wg^T) * (X Wu^T)``, and its gradients (the probe
  backward of the calibration goes through it; a trained block wants ``dWg`` and ``dWu`` too);
* a frozen projection in 4 bits with group scales for a few tokens, with each token's adapter beside
  it: ``Y = X W^T + s_a (X A_a) B_a^T``, ``W = scale (code - zero)``.

``run`` computes them in plain torch operations (``own = False``) or through this repository's
library (``own = True``).  Widths are those of the synthetic workloads (896, 2048, 3584, 5120) and
four times as much in the feed-forward; vocabularies of 49152 and 151936, ranks 8 to 32.
"""

import math

import torch

own = False


def listed():
    return [
        # scoring a few answers of a student against its teacher: latency, the head is read once
        dict(name="distill_score", op="distill", n=37, d=2048, v=49152, k=16, masked=0.0, short=0.0, tau=1.0, weights=False,
             dh=False, dw=False),
        # probe backward of a calibration that follows a teacher: frozen head, hidden-state gradients
        dict(name="distill_probe", op="distill", n=1531, d=3584, v=151936, k=64, masked=0.0, short=0.2, tau=1.0, weights=False,
             dh=True, dw=False),
        # a training step with a trained head: prompts masked, weighted positions, softened teacher
        dict(name="distill_train", op="distill", n=4096, d=2048, v=49152, k=32, masked=0.25, short=0.1, tau=2.0, weights=True,
             dh=True, dw=True),
        # a ragged small model: odd token count, odd vocabulary, few logits a position
        dict(name="distill_ragged", op="distill", n=777, d=896, v=32003, k=5, masked=0.1, short=0.5, tau=1.5, weights=True,
             dh=True, dw=True),
        # one token through a block: latency, both weights are read once
        dict(name="gated_token", op="gated", n=1, d=3584, f=14336, act="silu", dx=False, dw=False),
        # a decoding step of 64 requests
        dict(name="gated_decode", op="gated", n=64, d=2048, f=8192, act="silu", dx=False, dw=False),
        # prompts
        dict(name="gated_prompt", op="gated", n=8192, d=3584, f=14336, act="silu", dx=False, dw=False),
        # probe backward through a frozen block: an odd number of tokens
        dict(name="gated_probe", op="gated", n=1531, d=5120, f=13656, act="gelu", dx=True, dw=False),
        # a training step of one block
        dict(name="gated_train", op="gated", n=4096, d=2048, f=8192, act="silu", dx=True, dw=True),
        # one token of one request, its adapter beside the 4-bit projection
        dict(name="q4_token", op="q4", n=1, d=3584, o=3584, group=128, zeros=False, f32=False, k=16, a=4),
        # a small batch of decoding requests over a wide projection, an adapter each
        dict(name="q4_decode", op="q4", n=8, d=5120, o=20480, group=64, zeros=True, f32=False, k=32, a=8),
        # a batch against the vocabulary head, an odd number of rows, no adapters, fp32 scales
        dict(name="q4_head", op="q4", n=3, d=2048, o=151931, group=32, zeros=True, f32=True, k=0, a=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["distill", "gated", "q4"])
    if op == "distill":
        d, v = 8 * _log(rng, 64, 640), _log(rng, 1000, 151936)
        dh = rng.random() < 0.6
        n = max(1, min(_log(rng, 1, 16384), int(2.5e11 / (d * v))))
        return dict(op=op, n=n, d=d, v=v, k=_log(rng, 1, 128), masked=rng.choice([0.0, 0.1, 0.5, 0.9]),
                    short=rng.choice([0.0, 0.3]), tau=rng.choice([0.7, 1.0, 2.0, 4.0]), weights=rng.random() < 0.5, dh=dh,
                    dw=dh and rng.random() < 0.6)
    if op == "gated":
        d, f = 8 * _log(rng, 64, 640), 8 * _log(rng, 64, 2560)
        dx = rng.random() < 0.6
        n = max(1, min(_log(rng, 1, 16384), int((1.3e11 if dx else 4.0e11) / (d * f))))
        return dict(op=op, n=n, d=d, f=f, act=rng.choice(["silu", "gelu"]), dx=dx, dw=dx and rng.random() < 0.6)
    group, k = rng.choice([32, 64, 128]), rng.choice([0, 0, 4, 8, 16, 24, 32, 64])
    d = group * max(1, _log(rng, 256, 8192) // group)
    return dict(op=op, n=_log(rng, 1, 64), d=d, o=8 * _log(rng, 32, 8192) if k else _log(rng, 250, 65536), group=group,
                zeros=rng.random() < 0.5, f32=rng.random() < 0.5, k=k, a=_log(rng, 1, 64) if k else 0)


def work(case):
    n = case["n"]
    if case["op"] == "distill":
        d, v = case["d"], case["v"]
        live = max(1, round(n * (1.0 - case["masked"])))  # a masked position needs no product
        products = 1 + int(case["dh"]) + int(case["dw"])
        nbytes = 2 * live * d + 2 * v * d + 8 * n * case["k"] + 8 * n + 2 * n * d * int(case["dh"]) + 2 * v * d * int(case["dw"])
        return {"bytes": nbytes, "flops": 2 * live * d * v * products}
    if case["op"] == "gated":
        d, f = case["d"], case["f"]
        nbytes = 2 * n * d + 4 * d * f + 2 * n * f
        flops = 4 * n * d * f
        if case["dx"]:
            nbytes += 2 * n * f + 2 * n * d
            flops += 4 * n * d * f
        if case["dw"]:
            nbytes += 4 * d * f
            flops += 4 * n * d * f
        return {"bytes": nbytes, "flops": flops}
    d, o, k = case["d"], case["o"], case["k"]
    groups = o * (d // case["group"])
    used = min(n, case["a"])
    nbytes = o * d // 2 + groups * ((4 if case["f32"] else 2) + int(case["zeros"])) + 2 * n * (d + o) + 2 * used * k * (d + o)
    return {"bytes": nbytes, "flops": 2 * n * (d * o + k * (d + o))}


def _gen(seed, case):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * int(seed) + sum(int(1000 * x) for x in case.values() if isinstance(x, (int, float))))
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _distill_inputs(case, seed):
    g = _gen(seed, case)
    n, d, v, k = case["n"], case["d"], case["v"], case["k"]
    s = {"case": case}
    W = _randn(g, v, d, scale=2.0 / math.sqrt(d), dtype=torch.bfloat16)
    # K words of each position, no word twice, in the order of the teacher's logits (largest first)
    first = torch.randint(0, v, (n, 1), generator=g, device="cuda")
    step = torch.randint(1, max(2, v // k), (n, 1), generator=g, device="cuda")
    idx = (first + step * _rand(g, n, k).argsort(1)) % v
    rank = torch.arange(k, device="cuda", dtype=torch.float32)
    s["t"] = (9.0 - 2.0 * torch.log1p(rank) + 0.3 * torch.randn((n, k), generator=g, device="cuda")).sort(1, descending=True)[0]
    # the student leans towards the teacher's first words, about half of the positions strongly
    lean = 0.5 + 2.0 * (_rand(g, n, 1) < 0.5).float()
    H = _randn(g, n, d)
    for j in range(min(3, k)):
        H += lean / (1 + j) * W[idx[:, j]].float()
    s["H"], s["W"] = H.to(torch.bfloat16), W
    # some teachers give fewer words, masked positions none
    keep = torch.where(_rand(g, n, 1) < case["short"], 1 + (k * _rand(g, n, 1)).floor(), torch.full((n, 1), float(k), device="cuda"))
    keep = torch.where(_rand(g, n, 1) < case["masked"], 0.0, keep)
    s["idx"] = torch.where(rank < keep, idx, -1).to(torch.int32)
    s["w"] = _rand(g, n) + 0.5 if case["weights"] else None
    return s


def _gated_inputs(case, seed):
    g = _gen(seed, case)
    n, d, f = case["n"], case["d"], case["f"]
    s = {"case": case, "X": _randn(g, n, d, dtype=torch.bfloat16)}
    s["Wg"] = _randn(g, f, d, scale=1.0 / math.sqrt(d), dtype=torch.bfloat16)
    s["Wu"] = _randn(g, f, d, scale=1.0 / math.sqrt(d), dtype=torch.bfloat16)
    if case["dx"]:
        s["dH"] = _randn(g, n, f, scale=0.01, dtype=torch.bfloat16)
    return s


def _q4_inputs(case, seed):
    g = _gen(seed, case)
    n, d, o, k, a, groups = case["n"], case["d"], case["o"], case["k"], case["a"], case["d"] // case["group"]
    s = {"case": case, "X": _randn(g, n, d, dtype=torch.bfloat16)}
    s["codes"] = torch.randint(0, 256, (o, d // 2), generator=g, device="cuda", dtype=torch.uint8)  # even k in the low half
    s["scales"] = ((0.5 + _rand(g, o, groups)) / (4.6 * math.sqrt(d))).to(torch.float32 if case["f32"] else torch.bfloat16)
    s["zeros"] = torch.randint(6, 11, (o, groups), generator=g, device="cuda", dtype=torch.uint8) if case["zeros"] else None
    if k:
        s["A"] = _randn(g, a, d, k, scale=1.0 / math.sqrt(d), dtype=torch.bfloat16)
        s["B"] = _randn(g, a, o, k, scale=0.3 / math.sqrt(k), dtype=torch.bfloat16)
        s["scale"] = 0.5 + _rand(g, a)
        ids = torch.randperm(a, generator=g, device="cuda")[torch.arange(n, device="cuda") % a]
        s["ids"] = torch.where(_rand(g, n) < 0.1, -1, ids).to(torch.int32)
    return s


def prepare(case, seed):
    n, d = case["n"], case["d"]
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    if case["op"] == "distill":
        s = _distill_inputs(case, seed)
        v, k = case["v"], case["k"]
        s["loss"], s["lse"] = torch.empty((n,), device="cuda"), torch.empty((n,), device="cuda")
        s["dH"] = torch.empty((n, d), **bf16) if case["dh"] else None
        s["dW"] = torch.empty((v, d), **bf16) if case["dw"] else None
        if own:  # the scratch memory that a program keeps
            from paper_2608_03020_gb300 import loca

            nbytes = loca.head_distill_workspace_size(n, v, d, k)
            if case["dh"]:
                nbytes = max(nbytes, loca.head_distill_backward_workspace_size(n, v, d, k, case["dh"], case["dw"]))
            s["ws"] = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
        return s
    if case["op"] == "gated":
        s = _gated_inputs(case, seed)
        f = case["f"]
        s["H"] = torch.empty((n, f), **bf16)
        s["dX"] = torch.empty((n, d), **bf16) if case["dx"] else None
        s["dWg"] = torch.empty((f, d), **bf16) if case["dw"] else None
        s["dWu"] = torch.empty((f, d), **bf16) if case["dw"] else None
        if own:
            from paper_2608_03020_gb300 import loca

            nbytes = loca.gated_workspace_size(n, d, f)
            if case["dx"]:
                nbytes = max(nbytes, loca.gated_backward_workspace_size(n, d, f, True, case["dw"]))
            s["ws"] = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
        return s
    s = _q4_inputs(case, seed)
    s["Y"] = torch.empty((n, case["o"]), **bf16)
    if own:  # the weight's and the adapters' device layouts, the step's token plan, scratch memory
        from paper_2608_03020_gb300 import loca

        s["weight"] = loca.Q4Weight(s["codes"], s["scales"], zeros=s["zeros"])
        s["set"] = s["plan"] = None
        if case["k"]:
            s["set"] = loca.AdapterSet(case["a"], d, case["o"], case["k"]).pack(s["A"], s["B"], s["scale"])
            s["plan"] = loca.AdapterPlan(s["ids"], case["a"])
        nbytes = loca.q4_workspace_size(n, d, case["o"], case["k"], case["a"])
        s["ws"] = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
    return s


def _distill_plain(s):
    case, W, tau = s["case"], s["W"].float(), s["case"]["tau"]
    idx, w = s["idx"].long(), s["w"]
    has = idx >= 0
    live = has.any(1)
    H = torch.where(live[:, None], s["H"].float(), 0.0)
    z = (H @ W.T) / tau
    top = z.amax(1, keepdim=True)
    zk = z.gather(1, torch.where(has, idx, 0))
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    t = torch.where(has, s["t"] / tau, -math.inf)
    t = t - torch.where(live[:, None], t.amax(1, keepdim=True), 0.0)
    q = torch.exp(t)
    mass = torch.where(live[:, None], q.sum(1, keepdim=True), 1.0)
    q = q / mass
    weight = live.float() if w is None else torch.where(live, w, 0.0)
    gap = (t - torch.log(mass)) - ((zk - top) - torch.log(total))
    loss = weight * tau * tau * torch.where(q > 0, q * gap, 0.0).sum(1)
    got = {"loss": loss, "lse": torch.where(live, lse, 0.0)}
    if case["dh"]:
        del z
        dz = p.div_(total)
        dz.scatter_add_(1, torch.where(has, idx, 0), -q)
        dz.mul_(tau * weight[:, None])
        scale = 1.0 / case["n"]
        got["dH"] = (scale * (dz @ W)).to(torch.bfloat16)
        if case["dw"]:
            got["dW"] = (scale * (dz.T @ H)).to(torch.bfloat16)
    return got


def _act_plain(name, g):
    """The activation and its derivative."""
    if name == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    c = math.sqrt(2.0 / math.pi)  # the tanh form
    th = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * c * (1.0 + 3.0 * 0.044715 * g * g)


def _gated_plain(s):
    case = s["case"]
    X, Wg, Wu = s["X"].float(), s["Wg"].float(), s["Wu"].float()
    gate, up = X @ Wg.T, X @ Wu.T
    a, da = _act_plain(case["act"], gate)
    got = {"H": (a * up).to(torch.bfloat16)}
    if case["dx"]:
        dH = s["dH"].float()
        dg, du = dH * up * da, dH * a
        got["dX"] = (dg @ Wg + du @ Wu).to(torch.bfloat16)
        if case["dw"]:
            got["dWg"], got["dWu"] = (dg.T @ X).to(torch.bfloat16), (du.T @ X).to(torch.bfloat16)
    return got


def _q4_weight(s, dtype):
    """The values that the codes stand for."""
    case, codes = s["case"], s["codes"]
    o, d = case["o"], case["d"]
    q = torch.stack([codes & 15, codes >> 4], 2).reshape(o, d // case["group"], case["group"]).to(dtype)
    zero = 8.0 if s["zeros"] is None else s["zeros"].to(dtype)[:, :, None]
    return (s["scales"].to(dtype)[:, :, None] * (q - zero)).reshape(o, d)


def _q4_plain(s):
    X = s["X"].float()
    y = X @ _q4_weight(s, torch.float32).T
    if s["case"]["k"]:
        case, ids = s["case"], s["ids"].long()
        a, k = case["a"], case["k"]
        A = s["A"].float().permute(1, 0, 2).reshape(case["d"], a * k)
        B = (s["B"].float() * s["scale"][:, None, None]).permute(1, 0, 2).reshape(case["o"], a * k)
        mine = (ids[:, None] == torch.arange(a, device="cuda")[None, :]).float().repeat_interleave(k, 1)
        y = y + ((X @ A) * mine) @ B.T
    return {"Y": y.to(torch.bfloat16)}


def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "distill":
            return _distill_plain(s)
        if case["op"] == "gated":
            return _gated_plain(s)
        return _q4_plain(s)
    from paper_2608_03020_gb300 import loca

    if case["op"] == "distill":
        loca.loca_head_distill(s["H"], s["W"], s["idx"], s["t"], s["loss"], lse=s["lse"], w=s["w"], tau=case["tau"],
                               workspace=s["ws"])
        got = {"loss": s["loss"], "lse": s["lse"]}
        if case["dh"]:
            loca.loca_head_distill_backward(s["H"], s["W"], s["idx"], s["t"], s["lse"], dH=s["dH"], dW=s["dW"], w=s["w"],
                                            tau=case["tau"], grad_scale=1.0 / case["n"], workspace=s["ws"])
            got["dH"] = s["dH"]
            if case["dw"]:
                got["dW"] = s["dW"]
        return got
    if case["op"] == "gated":
        loca.loca_gated(s["X"], s["Wg"], s["Wu"], s["H"], act=case["act"], workspace=s["ws"])
        got = {"H": s["H"]}
        if case["dx"]:
            loca.loca_gated_backward(s["X"], s["Wg"], s["Wu"], s["dH"], dX=s["dX"], dWg=s["dWg"], dWu=s["dWu"],
                                     act=case["act"], workspace=s["ws"])
            got["dX"] = s["dX"]
            if case["dw"]:
                got["dWg"], got["dWu"] = s["dWg"], s["dWu"]
        return got
    loca.loca_q4_apply(s["X"], s["weight"], s["Y"], adapters=s["set"], plan=s["plan"], workspace=s["ws"])
    return {"Y": s["Y"]}


def _distill_exact(case, seed):
    s = _distill_inputs(case, seed)
    n, d, tau = case["n"], case["d"], case["tau"]
    W = s["W"].double()
    f64 = dict(dtype=torch.float64, device="cuda")
    got = {"loss": torch.zeros((n,), **f64), "lse": torch.zeros((n,), **f64)}
    if case["dh"]:
        got["dH"] = torch.zeros((n, d), **f64)
    if case["dw"]:
        got["dW"] = torch.zeros((case["v"], d), **f64)
    for rows in torch.nonzero((s["idx"] >= 0).any(1))[:, 0].split(2048):
        idx = s["idx"][rows].long()
        H = s["H"][rows].double()
        w = torch.ones((len(rows),), **f64) if s["w"] is None else s["w"][rows].double()
        logp = torch.log_softmax(H @ W.T / tau, 1)
        logq = torch.log_softmax(torch.where(idx >= 0, s["t"][rows].double() / tau, -math.inf), 1)
        at = idx.clamp(min=0)
        each = logq.exp() * (logq - logp.gather(1, at))
        got["loss"][rows] = w * tau ** 2 * torch.where(idx >= 0, each, 0.0).sum(1)
        # log p of a word is its scaled logit minus the normaliser
        word = at[:, 0]
        got["lse"][rows] = (H * W[word]).sum(1) / tau - logp[torch.arange(len(rows), device="cuda"), word]
        if case["dh"]:
            error = logp.exp_().scatter_add_(1, at, -torch.where(idx >= 0, logq.exp(), 0.0)) * (w[:, None] * tau / n)
            got["dH"][rows] = error @ W
            if case["dw"]:
                got["dW"] += error.T @ H
    return got


def _gated_exact(case, seed):
    s = _gated_inputs(case, seed)
    X, Wg, Wu = s["X"].double(), s["Wg"].double(), s["Wu"].double()
    got = {}
    parts = {"H": [], "dX": []}
    if case["dw"]:
        got["dWg"], got["dWu"] = torch.zeros_like(Wg), torch.zeros_like(Wu)
    for r in range(0, case["n"], 4096):
        x = X[r:r + 4096]
        with torch.enable_grad():
            gate, up = (x @ Wg.T).requires_grad_(), (x @ Wu.T).requires_grad_()
            if case["act"] == "silu":
                h = torch.nn.functional.silu(gate) * up
            else:
                h = torch.nn.functional.gelu(gate, approximate="tanh") * up
            if case["dx"]:
                dg, du = torch.autograd.grad(h, (gate, up), s["dH"][r:r + 4096].double())
        parts["H"].append(h.detach())
        if case["dx"]:
            parts["dX"].append(dg @ Wg + du @ Wu)
        if case["dw"]:
            got["dWg"] += dg.T @ x
            got["dWu"] += du.T @ x
    got.update({name: torch.cat(p) for name, p in parts.items() if p})
    return got


def _q4_exact(case, seed):
    s = _q4_inputs(case, seed)
    X = s["X"].double()
    y = X @ _q4_weight(s, torch.float64).T
    for i in range(case["n"] if case["k"] else 0):
        a = int(s["ids"][i])
        if a >= 0:
            y[i] += s["scale"][a].double() * (s["B"][a].double() @ (X[i] @ s["A"][a].double()))
    return {"Y": y}


def exact(case, seed):
    return {"distill": _distill_exact, "gated": _gated_exact, "q4": _q4_exact}[case["op"]](case, seed)
