"""Timing cases of the training-step operators: embedding lookup, layer / RMS norm, and the loss over a
large vocabulary, each with its gradient.

`run` computes a case either in its plain form (elementary torch operations in 32 bits, rounded once at the
end) or, where `own` is set, through the library's entry points.  Sizes are those of the repository's two
model shapes (hidden 4096 and 2048, vocabulary 151936, whole or cut over TP receivers, head_dim 128) and
generic odd ones around them."""
import math

import torch

own = False

VOCAB = 151936
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------

def _lookup(tokens, hidden, rows, row_start, table, out):
    return dict(op="lookup", tokens=tokens, hidden=hidden, rows=rows, row_start=row_start, table=table, out=out)


def _lookup_grad(tokens, hidden, rows, row_start, dout, dtable):
    return dict(op="lookup_grad", tokens=tokens, hidden=hidden, rows=rows, row_start=row_start, dout=dout, dtable=dtable)


def _norm(op, rows, hidden, dtype, rms):
    return dict(op=op, rows=rows, hidden=hidden, dtype=dtype, rms=rms)


def _loss(op, tokens, ignored, hidden, vocab, vocab_start, scale):
    return dict(op=op, tokens=tokens, ignored=ignored, hidden=hidden, vocab=vocab, vocab_start=vocab_start, scale=scale)


def listed():
    return [
        # one decoding step of a batch of eight sequences: latency
        dict(_lookup(8, 4096, VOCAB, 0, "bf16", "bf16"), name="lookup-decode"),
        # the input layer of one training micro-batch
        dict(_lookup(16384, 4096, VOCAB, 0, "bf16", "bf16"), name="lookup-train"),
        # its gradient: dense fp32 gradient of the master embedding, token frequencies as text has them
        dict(_lookup_grad(16384, 4096, VOCAB, 0, "bf16", "fp32"), name="lookup-grad-train"),
        # the gradient of one of four vocabulary shards: most tokens belong to other ranks; odd count
        dict(_lookup_grad(6007, 2048, VOCAB // 4, VOCAB // 4, "fp32", "fp32"), name="lookup-grad-shard"),
        # a norm in front of the sampling head while decoding: latency
        dict(_norm("norm", 8, 4096, "bf16", False), name="norm-decode"),
        # a norm of a training micro-batch, fp32 residual stream, odd number of tokens
        dict(_norm("norm", 8191, 4096, "fp32", False), name="norm-train"),
        # its gradient in bf16
        dict(_norm("norm_grad", 16384, 4096, "bf16", False), name="norm-grad-train"),
        # per-head RMS norm of the queries (32 heads of 128), gradient
        dict(_norm("norm_grad", 8191 * 32, 128, "bf16", True), name="head-norm-grad"),
        # log-probabilities of one new token of eight sequences, as a sampler or a scorer asks for them
        dict(_loss("loss", 8, 0, 4096, VOCAB, 0, 1.0), name="logprob-decode"),
        # log-probabilities of rollouts before an RL step: prompts carry no loss; sampling temperature 0.7
        dict(_loss("loss", 8192, 2048, 4096, VOCAB, 0, 1.0 / 0.7), name="logprob-rollout"),
        # loss and gradients on one of four vocabulary shards, odd token count
        dict(_loss("loss_grad", 1021, 100, 2048, VOCAB // 4, VOCAB // 4, 1.0), name="loss-grad-shard"),
        # loss and gradients of a training micro-batch over the whole vocabulary: the largest
        dict(_loss("loss_grad", 8192, 0, 4096, VOCAB, 0, 1.0), name="loss-grad-train"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["lookup", "lookup_grad", "norm", "norm_grad", "loss", "loss_grad"])
    if op.startswith("lookup"):
        hidden = rng.choice([2048, 4096, 8 * rng.randint(16, 640), rng.randint(65, 3001)])
        parts = rng.choice([1, 1, 2, 4])
        rows = VOCAB // parts
        start = rows * rng.randrange(parts)
        tokens = log(1, 32768)
        a, b = rng.choice(["bf16", "fp32"]), rng.choice(["bf16", "fp32"])
        return (_lookup if op == "lookup" else _lookup_grad)(tokens, hidden, rows, start, a, b)
    if op.startswith("norm"):
        hidden = rng.choice([128, 128, 2048, 4096, 8 * rng.randint(8, 1024), rng.randint(33, 5001)])
        rows = min(log(1, 262144), (1 << 27) // hidden)
        return _norm(op, rows, hidden, rng.choice(["bf16", "fp32"]), rng.random() < 0.5)
    hidden = rng.choice([2048, 4096, 8 * rng.randint(16, 512)])
    parts = rng.choice([1, 2, 4])
    vocab = rng.choice([VOCAB // parts, rng.randint(1000, VOCAB)])
    tokens = log(1, 8192)
    ignored = int(tokens * rng.choice([0.0, 0.25, 0.6]))
    start = rng.choice([0, VOCAB - vocab])
    return _loss(op, tokens, ignored, hidden, vocab, start, rng.choice([1.0, 1.25]))


# ---- inputs ---------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _normal(g, shape, std, dtype, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def _token_ids(seed, n):
    """Ids over the whole vocabulary with the skewed frequencies of text (Zipf with an offset), shuffled.
    Drawn on the host: the same seed gives the same ids everywhere."""
    g = torch.Generator().manual_seed(seed)
    mass = (1.0 / (torch.arange(VOCAB, dtype=torch.float64) + 2.7)).cumsum(0)
    name = torch.randperm(VOCAB, generator=g)
    return name[torch.searchsorted(mass, torch.rand(n, dtype=torch.float64, generator=g) * mass[-1]).clamp_(max=VOCAB - 1)]


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": case}
    if op == "lookup":
        dt, do = DTYPES[case["table"]], DTYPES[case["out"]]
        s["table"] = _normal(g, (case["rows"], case["hidden"]), 0.02, dt)
        s["ids"] = _token_ids(seed, case["tokens"]).cuda()
        s["scale"] = math.sqrt(case["hidden"])
        s["out"] = torch.empty(case["tokens"], case["hidden"], dtype=do, device="cuda")
    elif op == "lookup_grad":
        s["dout"] = _normal(g, (case["tokens"], case["hidden"]), 1e-3, DTYPES[case["dout"]])
        s["ids"] = _token_ids(seed, case["tokens"]).cuda()
        s["scale"] = math.sqrt(case["hidden"])
        s["dtable"] = torch.empty(case["rows"], case["hidden"], dtype=DTYPES[case["dtable"]], device="cuda")
    elif op in ("norm", "norm_grad"):
        rows, hidden, dt, rms = case["rows"], case["hidden"], DTYPES[case["dtype"]], case["rms"]
        # a residual stream: activations with an offset and a few strong channels
        chan = torch.empty(hidden, device="cuda").normal_(0, 0.5, generator=g).exp()
        s["x"] = (_normal(g, (rows, hidden), 1.0, torch.float32, 0.1) * chan).to(dt)
        s["weight"] = _normal(g, (hidden,), 0.02, torch.float32, 1.0)
        s["bias"] = None if rms else _normal(g, (hidden,), 0.02, torch.float32)
        s["mean"] = None if rms else torch.empty(rows, device="cuda")
        s["rstd"] = torch.empty(rows, device="cuda")
        if op == "norm":
            s["out"] = torch.empty(rows, hidden, dtype=dt, device="cuda")
        else:
            x = s["x"].float()
            mean = x.mean(1)
            if not rms:
                s["mean"].copy_(mean)
                x = x - mean[:, None]
            s["rstd"].copy_((x.square().mean(1) + EPS).rsqrt())
            s["dout"] = _normal(g, (rows, hidden), 1e-3, dt)
            s["dx"] = torch.empty(rows, hidden, dtype=dt, device="cuda")
            s["dweight"] = torch.empty(hidden, device="cuda")
            s["dbias"] = None if rms else torch.empty(hidden, device="cuda")
    else:
        n, hidden, vocab = case["tokens"], case["hidden"], case["vocab"]
        s["x"] = _normal(g, (n, hidden), 1.5, torch.bfloat16)
        s["weight"] = _normal(g, (vocab, hidden), 0.8 / math.sqrt(hidden), torch.bfloat16)
        t = _token_ids(seed, n)
        t[torch.randperm(n, generator=torch.Generator().manual_seed(seed + 1))[:case["ignored"]]] = -100
        s["targets"] = t.cuda()
        for k in ("lse", "target_logit", "loss"):
            s[k] = torch.empty(n, device="cuda")
        if op == "loss_grad":
            # advantage-weighted mean over the tokens that count
            s["dloss"] = torch.empty(n, device="cuda").normal_(0, 1, generator=g) / max(1, n - case["ignored"])
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"] = torch.empty_like(s["weight"])
    return s


# ---- one pass -------------------------------------------------------------------------------------

def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op in ("lookup", "lookup_grad"):
        local = s["ids"] - c["row_start"]
        here = (local >= 0) & (local < c["rows"])
        local = torch.where(here, local, 0)
        if op == "lookup":
            y = s["table"][local].float() * s["scale"]
            return {"out": (y * here[:, None]).to(s["out"].dtype)}
        d = s["dout"].float() * (here * s["scale"])[:, None]
        e = torch.zeros(c["rows"], c["hidden"], device="cuda").index_add_(0, local, d)
        return {"dtable": e.to(s["dtable"].dtype)}
    if op == "norm":
        x = s["x"].float()
        mean = None
        if not c["rms"]:
            mean = x.mean(1)
            x = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        y = x * rstd[:, None] * s["weight"]
        if s["bias"] is not None:
            y = y + s["bias"]
        return {"out": y.to(s["out"].dtype), "mean": mean, "rstd": rstd} if mean is not None else {"out": y.to(s["out"].dtype), "rstd": rstd}
    if op == "norm_grad":
        x, dy = s["x"].float(), s["dout"].float()
        if not c["rms"]:
            x = x - s["mean"][:, None]
        xhat = x * s["rstd"][:, None]
        g = dy * s["weight"]
        dx = g - xhat * (g * xhat).mean(1, keepdim=True)
        if not c["rms"]:
            dx = dx - g.mean(1, keepdim=True)
        r = {"dx": (dx * s["rstd"][:, None]).to(s["dx"].dtype), "dweight": (dy * xhat).sum(0)}
        if not c["rms"]:
            r["dbias"] = dy.sum(0)
        return r
    x, w = s["x"].float(), s["weight"].float()
    t = s["targets"]
    keep = t >= 0
    local = t - c["vocab_start"]
    here = keep & (local >= 0) & (local < c["vocab"])
    local = torch.where(here, local, 0)
    logits = (x @ w.T).mul_(c["scale"])
    top = logits.amax(1, keepdim=True)
    at = torch.where(here, logits.gather(1, local[:, None])[:, 0], 0.0)
    p = logits.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    lse = torch.where(keep, (top + total.log())[:, 0], 0.0)
    r = {"lse": lse, "target_logit": at, "loss": torch.where(keep, lse - at, 0.0)}
    if op == "loss_grad":
        f = torch.where(keep, s["dloss"], 0.0) * c["scale"]
        p.mul_(f[:, None] / total)
        p.scatter_add_(1, local[:, None], -(f * here)[:, None])
        r["dx"] = (p @ w).to(s["dx"].dtype)
        r["dweight"] = (p.T @ x).to(s["dweight"].dtype)
    return r


def _workspace(s, nbytes):
    ws = s.get("workspace")
    if ws is None:  # kept with the state, as a program keeps it from call to call
        ws = s["workspace"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
    return ws


def _library(s):
    import paper_2608_00455_b200 as dte

    c, op = s["case"], s["case"]["op"]
    if op == "lookup":
        dte.dte_embedding_forward(s["table"], s["ids"], s["out"], scale=s["scale"], row_start=c["row_start"], vocab=VOCAB)
        return {"out": s["out"]}
    if op == "lookup_grad":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, dte.dte_embedding_backward_workspace_bytes(c["tokens"], c["hidden"]))
        dte.dte_embedding_backward(s["dout"], s["ids"], s["dtable"], ws, scale=s["scale"], row_start=c["row_start"], vocab=VOCAB)
        return {"dtable": s["dtable"]}
    if op == "norm":
        dte.dte_norm_forward(s["x"], s["weight"], s["bias"], s["out"], s["mean"], s["rstd"], EPS, rms=c["rms"])
        return {"out": s["out"], "rstd": s["rstd"]} if c["rms"] else {"out": s["out"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_grad":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, dte.dte_norm_backward_workspace_bytes(c["rows"], c["hidden"]))
        dte.dte_norm_backward(s["dout"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"], ws, rms=c["rms"])
        return {"dx": s["dx"], "dweight": s["dweight"]} if c["rms"] else {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
    ws = s.get("workspace")
    if ws is None:
        size = dte.dte_linear_ce_forward_workspace_bytes(c["tokens"], c["vocab"], c["hidden"])
        if op == "loss_grad":
            size = max(size, dte.dte_linear_ce_backward_workspace_bytes(c["tokens"], c["vocab"], c["hidden"]))
        ws = _workspace(s, size)
    dte.dte_linear_ce_forward(s["x"], s["weight"], s["targets"], s["lse"], s["target_logit"], s["loss"], ws,
                              logit_scale=c["scale"], vocab_start=c["vocab_start"], vocab=VOCAB)
    r = {"lse": s["lse"], "target_logit": s["target_logit"], "loss": s["loss"]}
    if op == "loss_grad":
        dte.dte_linear_ce_backward(s["x"], s["weight"], s["targets"], s["lse"], s["dloss"], s["dx"], s["dweight"], ws,
                                   logit_scale=c["scale"], vocab_start=c["vocab_start"], vocab=VOCAB)
        r["dx"], r["dweight"] = s["dx"], s["dweight"]
    return r


def run(state):
    return _library(state) if own else _plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    op = case["op"]
    if op == "lookup":
        # the share of the tokens that this shard holds, once each (distinct rows are fewer: at most this)
        n, h = case["tokens"], case["hidden"]
        share = case["rows"] / VOCAB
        return {"bytes": n * 8 + n * share * h * _size(case["table"]) + n * h * _size(case["out"]), "flops": n * share * h}
    if op == "lookup_grad":
        n, h = case["tokens"], case["hidden"]
        share = case["rows"] / VOCAB
        return {"bytes": n * 8 + n * share * h * _size(case["dout"]) + case["rows"] * h * _size(case["dtable"]), "flops": n * share * h}
    if op in ("norm", "norm_grad"):
        r, h, b = case["rows"], case["hidden"], _size(case["dtype"])
        stats = r * 4 * (1 if case["rms"] else 2)
        if op == "norm":
            return {"bytes": 2 * r * h * b + stats + h * 4 * (1 if case["rms"] else 2), "flops": 8 * r * h}
        return {"bytes": 3 * r * h * b + stats + h * 4 * (2 if case["rms"] else 3), "flops": 12 * r * h}
    n, h, v = case["tokens"], case["hidden"], case["vocab"]
    m = n - case["ignored"]
    if op == "loss":
        return {"bytes": 2 * (m * h + v * h) + n * 20, "flops": 2 * m * v * h}
    return {"bytes": 2 * (m * h + n * h + 2 * v * h) + n * 24, "flops": 6 * m * v * h}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    dbl = torch.float64
    if op == "lookup":
        out = torch.zeros(case["tokens"], case["hidden"], dtype=dbl, device="cuda")
        mine = ((s["ids"] >= case["row_start"]) & (s["ids"] < case["row_start"] + case["rows"])).nonzero()[:, 0]
        out[mine] = s["table"].index_select(0, s["ids"][mine] - case["row_start"]).to(dbl) * s["scale"]
        return {"out": out}
    if op == "lookup_grad":
        # sums per distinct token, from the sorted ids and differences of running sums in blocks of columns
        out = torch.zeros(case["rows"], case["hidden"], dtype=dbl, device="cuda")
        mine = ((s["ids"] >= case["row_start"]) & (s["ids"] < case["row_start"] + case["rows"])).nonzero()[:, 0]
        if mine.numel():
            ids, order = s["ids"][mine].sort()
            row, count = ids.unique_consecutive(return_counts=True)
            last = count.cumsum(0) - 1
            for c in range(0, case["hidden"], 512):
                run_sum = s["dout"][mine[order], c:c + 512].to(dbl).cumsum(0)[last]
                run_sum[1:] -= run_sum[:-1].clone()
                out[row - case["row_start"], c:c + 512] = run_sum * s["scale"]
        return {"dtable": out}
    if op == "norm":
        x = s["x"].to(dbl)
        r = {}
        centre = 0.0
        if not case["rms"]:
            centre = x.sum(1, keepdim=True) / case["hidden"]
            r["mean"] = centre[:, 0]
        power = ((x - centre) ** 2).sum(1, keepdim=True) / case["hidden"]
        r["rstd"] = (power + EPS)[:, 0] ** -0.5
        r["out"] = (x - centre) / (power + EPS).sqrt() * s["weight"].to(dbl) + (0.0 if case["rms"] else s["bias"].to(dbl))
        return r
    if op == "norm_grad":
        rows, h = case["rows"], case["hidden"]
        w = s["weight"].to(dbl)
        dx = torch.empty(rows, h, dtype=dbl, device="cuda")
        dw, db = torch.zeros(h, dtype=dbl, device="cuda"), torch.zeros(h, dtype=dbl, device="cuda")
        for a in range(0, rows, 65536):
            b = slice(a, a + 65536)
            u = s["x"][b].to(dbl) - (0.0 if case["rms"] else s["mean"][b, None].to(dbl))
            k = s["rstd"][b, None].to(dbl)
            dy = s["dout"][b].to(dbl)
            dw += torch.einsum("rh,rh->h", dy, u * k)
            db += dy.sum(0)
            # derivative of u * k with k a function of u
            d = k * dy * w - k ** 3 * u * torch.einsum("rh,rh->r", dy * w, u)[:, None] / h
            dx[b] = d if case["rms"] else d - k * (dy @ w)[:, None] / h
        return {"dx": dx, "dweight": dw} if case["rms"] else {"dx": dx, "dweight": dw, "dbias": db}
    n, h, v = case["tokens"], case["hidden"], case["vocab"]
    if 6.0 * n * h * v > 4e14:
        return None
    w = s["weight"].to(dbl)
    out = {k: torch.zeros(n, dtype=dbl, device="cuda") for k in ("lse", "target_logit", "loss")}
    grad = op == "loss_grad"
    if grad:
        out["dx"] = torch.zeros(n, h, dtype=dbl, device="cuda")
        out["dweight"] = torch.zeros(v, h, dtype=dbl, device="cuda")
    counted = (s["targets"] >= 0).nonzero()[:, 0]
    for a in range(0, counted.numel(), 1024):
        at = counted[a:a + 1024]
        x = s["x"][at].to(dbl)
        z = case["scale"] * torch.mm(x, w.t())
        out["lse"][at] = torch.logsumexp(z, 1)
        col = s["targets"][at] - case["vocab_start"]
        row = ((col >= 0) & (col < v)).nonzero()[:, 0]
        out["target_logit"][at[row]] = z[row, col[row]]
        out["loss"][at] = out["lse"][at] - out["target_logit"][at]
        if grad:
            z = torch.softmax(z, 1)
            z[row, col[row]] -= 1.0
            z *= (s["dloss"][at].to(dbl) * case["scale"])[:, None]
            out["dx"][at] = torch.mm(z, w)
            out["dweight"].addmm_(z.t(), x)
    return out
