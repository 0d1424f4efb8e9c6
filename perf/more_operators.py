"""Timing cases of the training step's middle and its end: rotary positions, causal attention over packed prompts
(grouped heads, sequences of different lengths), each with its gradient, and the global gradient norm with clipping.

`run` computes a case either in its plain form (elementary torch operations in 32 bits, angles in 64, rounded once
at the end) or, where `own` is set, through the library's entry points.  Heads are those of the repository's two model
shapes (32 query heads on 8 or 4 key heads of 128), gradients those of one layer of each; the other sizes are generic."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
ROPE_BASE = 1e6
YARN = dict(factor=4.0, original=32768, fast=32.0, slow=1.0)


# ---- cases ----------------------------------------------------------------------------------------

def _rope(tokens, heads, kv_heads, head_dim, rot, interleaved, dtype, far, inverse, fused):
    return dict(op="rope", tokens=tokens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, rot=rot, interleaved=interleaved,
                dtype=dtype, far=far, inverse=inverse, fused=fused)


def _attention(op, tokens, sequences, spread, behind, heads, kv_heads, head_dim, fused):
    """`tokens` rows cut into `sequences` lengths that differ by about a factor e^(2 spread); `behind` rows follow
    the last sequence and belong to none."""
    return dict(op=op, tokens=tokens, sequences=sequences, spread=spread, behind=behind, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, fused=fused)


def _clip(shapes, copies, dtype, out, times):
    """`copies` times the gradients in `shapes` ("rows x cols" separated by commas); the norm comes out near `times` the largest allowed."""
    return dict(op="clip", shapes=shapes, copies=copies, dtype=dtype, out=out, times=times)


DENSE_LAYER = "1x4096,4096x4096,1024x4096,1024x4096,1x128,1x128,4096x4096,1x4096,12288x4096,12288x4096,4096x12288"
MOE_EXPERT = "768x2048,768x2048,2048x768"


def listed():
    return [
        # one decoding step of eight sequences far into a context extended by YaRN: latency
        dict(_rope(8, 32, 8, 128, 128, False, "bf16", True, False, False), name="rope-decode"),
        # queries and keys of a training micro-batch, cut out of one projection's output
        dict(_rope(16384, 32, 8, 128, 128, False, "bf16", False, False, True), name="rope-train"),
        # the gradient of interleaved pairs in half of each head, fp32, odd number of tokens
        dict(_rope(8191, 32, 4, 128, 64, True, "fp32", False, True, False), name="rope-grad-partial"),
        # one short prompt: latency
        dict(_attention("attention", 77, 1, 0.0, 0, 32, 8, 128, True), name="prompt-short"),
        # scoring a micro-batch of packed rollouts of ragged lengths, some padding behind them
        dict(_attention("attention", 8192, 19, 0.8, 61, 32, 4, 128, True), name="prompts-packed"),
        # one long document: the largest forward pass
        dict(_attention("attention", 32768, 1, 0.0, 0, 32, 8, 128, False), name="prompt-long"),
        # training on many short, uneven sequences, as many key heads as query heads, heads of 64
        dict(_attention("attention_grad", 4001, 57, 1.0, 5, 16, 16, 64, False), name="attention-grad-short"),
        # training on packed rollouts
        dict(_attention("attention_grad", 8192, 19, 0.8, 61, 32, 4, 128, True), name="attention-grad-packed"),
        # training on one long document: the largest
        dict(_attention("attention_grad", 16384, 1, 0.0, 0, 32, 8, 128, False), name="attention-grad-long"),
        # the norm weights and a slice of the projections of a layer, as a sharded optimizer holds them; no clipping: latency
        dict(_clip("1x4096,1x4096,1x128,1x128,256x4096,255x4096", 1, "bf16", "fp32", 0.8), name="clip-small"),
        # one of eight ranks' experts of a layer: many tensors
        dict(_clip(MOE_EXPERT, 16, "fp32", "fp32", 3.0), name="clip-experts"),
        # the gradients of five dense layers: the largest
        dict(_clip(DENSE_LAYER, 5, "bf16", "fp32", 3.0), name="clip-dense-layers"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rope", "attention", "attention", "attention_grad", "attention_grad", "clip"])
    if op == "rope":
        heads, kv = rng.choice([(32, 8), (32, 4), (16, 16), (5, 1)])
        dim = rng.choice([128, 128, 64, 2 * rng.randint(8, 128)])
        rot = dim if rng.random() < 0.5 else 2 * rng.randint(1, dim // 2)
        return _rope(log(1, 16384), heads, kv, dim, rot, rng.random() < 0.5, rng.choice(["bf16", "fp32"]), rng.random() < 0.5,
                     rng.random() < 0.5, rng.random() < 0.5)
    if op == "clip":
        shapes = ",".join(f"{log(1, 4096)}x{log(1, 4096)}" for _ in range(rng.randint(1, 12)))
        return _clip(shapes, rng.choice([1, 1, 3, rng.randint(1, 5)]), rng.choice(["bf16", "fp32"]), rng.choice(["bf16", "fp32"]),
                     rng.choice([0.5, 2.0, 50.0]))
    heads, kv = rng.choice([(32, 8), (32, 4), (16, 16), (8, 1), (6, 2), (9, 3)])
    tokens = log(1, 16384)
    sequences = min(tokens, log(1, 64))
    return _attention(op, tokens, sequences, rng.choice([0.0, 0.5, 1.0]), rng.choice([0, 0, rng.randint(1, 200)]), heads, kv,
                      rng.choice([128, 128, 64, 8 * rng.randint(2, 16)]), rng.random() < 0.5)


def _lengths(case):
    """Lengths of the packed sequences; the case alone decides them."""
    n, t = case["sequences"], case["tokens"]
    rng = random.Random(f"{n} {t} {case['spread']}")
    share = [math.exp(rng.gauss(0.0, case["spread"])) for _ in range(n)]
    left, out = t - n, []                      # one token each, the others by share
    total = sum(share)
    for s in share:
        k = int(round(left * s / total)) if total > 0 else 0
        k = max(0, min(left, k))
        out.append(1 + k)
        left -= k
        total -= s
    out[-1] += left
    return out


def _shapes(case):
    return [tuple(int(n) for n in s.split("x")) for s in case["shapes"].split(",")] * case["copies"]


# ---- inputs ---------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _normal(g, shape, std, dtype, mean=0.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def _heads(g, case, rows, dtype, std):
    """Queries, keys and values (rows, heads, head_dim), one buffer each or cut out of a projection's output."""
    hq, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    if case["fused"]:
        x = _normal(g, (rows, hq + 2 * hk, d), std, dtype)
        return x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    return tuple(_normal(g, (rows, h, d), std, dtype) for h in (hq, hk, hk))


def prepare(case, seed):
    g = _gen(seed)
    host = random.Random(seed)
    op = case["op"]
    s = {"case": case}
    if op == "rope":
        s["q"], s["k"], _ = _heads(g, case, case["tokens"], DTYPES[case["dtype"]], 1.0)
        if case["far"]:       # one token each of sequences anywhere in the extended context
            pos = [host.randrange(int(YARN["factor"] * YARN["original"])) for _ in range(case["tokens"])]
        else:                 # packed sequences, counted from 0 each
            pos, n = [], 0
            for _ in range(case["tokens"]):
                pos.append(n)
                n = 0 if host.random() < 1 / 700 else n + 1
        s["positions"] = torch.tensor(pos, dtype=torch.int64).cuda()
        freq, s["amplitude"] = _frequencies(case["rot"], case["far"])
        s["freq"] = freq.cuda()
        s["q_out"], s["k_out"] = (torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in (s["q"], s["k"]))
    elif op in ("attention", "attention_grad"):
        lengths = _lengths(case)
        rows, hq = case["tokens"] + case["behind"], case["heads"]
        # normalised queries and keys: unit size, a common direction in the keys
        s["q"], s["k"], s["v"] = _heads(g, case, rows, torch.bfloat16, 1.0)
        s["k"].copy_(s["k"].float() + _normal(g, (1, case["kv_heads"], case["head_dim"]), 0.5, torch.float32))
        s["scale"] = case["head_dim"] ** -0.5
        starts = [0]
        for n in lengths:
            starts.append(starts[-1] + n)
        s["bounds"] = starts
        s["starts"] = torch.tensor(starts, dtype=torch.int32).cuda()
        s["out"] = torch.zeros(rows, hq, case["head_dim"], dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros(hq, rows, device="cuda")
        if op == "attention_grad":
            forward = _plain_attention(s)
            s["out"].copy_(forward["out"])
            s["lse"].copy_(forward["lse"])
            s["dout"] = _normal(g, (rows, hq, case["head_dim"]), 1e-3, torch.bfloat16)
            for name, like in (("dq", "q"), ("dk", "k"), ("dv", "v")):
                s[name] = torch.zeros(s[like].shape, dtype=torch.bfloat16, device="cuda")
        if own:               # made once per packed batch, used by every layer's forward and backward pass
            import paper_2608_00455_b200 as dte

            s["plan"] = torch.empty(dte.dte_attention_plan_bytes(rows, len(lengths)), dtype=torch.uint8, device="cuda")
            dte.dte_attention_plan(s["starts"], rows, s["plan"])
    else:
        shapes = _shapes(case)
        # spread over magnitudes from tensor to tensor, as layers' gradients are
        s["grads"] = [_normal(g, shape, 10.0 ** host.uniform(-5, -3), DTYPES[case["dtype"]]) for shape in shapes]
        s["outs"] = [torch.empty(shape, dtype=DTYPES[case["out"]], device="cuda") for shape in shapes]
        size = math.sqrt(sum(float(t.double().square().sum()) for t in s["grads"]))
        s["max_norm"] = size / case["times"]
        s["sum_squares"] = torch.empty((), dtype=torch.float64, device="cuda")
        s["norm"] = torch.empty((), device="cuda")
    return s


def _frequencies(rot, extended):
    """Angle per position of each pair, and the amplitude of the rotated values; YaRN where the context is extended."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    freq = ROPE_BASE ** (-2.0 * i / rot)
    if not extended:
        return freq, 1.0
    # pair index whose wave turns `n` times over the original context
    def at(n):
        return rot * math.log(YARN["original"] / (n * 2 * math.pi)) / (2 * math.log(ROPE_BASE))

    lo, hi = max(0.0, math.floor(at(YARN["fast"]))), min(rot - 1.0, math.ceil(at(YARN["slow"])))
    ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
    return freq * (1.0 - ramp) + freq / YARN["factor"] * ramp, 0.1 * math.log(YARN["factor"]) + 1.0


# ---- one pass -------------------------------------------------------------------------------------

def _plain_rope(s):
    c = s["case"]
    rot = c["rot"]
    angle = s["positions"].double()[:, None] * s["freq"]
    cos = (angle.cos() * s["amplitude"]).float()[:, None]
    sin = (angle.sin() * s["amplitude"]).float()[:, None] * (-1.0 if c["inverse"] else 1.0)
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        y = x.clone()
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        lo, hi = a * cos - b * sin, b * cos + a * sin
        if c["interleaved"]:
            y[..., 0:rot:2], y[..., 1:rot:2] = lo, hi
        else:
            y[..., :rot // 2], y[..., rot // 2:rot] = lo, hi
        out[name] = y.to(s[name].dtype)
    return out


def _pieces(s):
    """(rows of a sequence, key head, its query heads)."""
    c = s["case"]
    group = c["heads"] // c["kv_heads"]
    for a, b in zip(s["bounds"], s["bounds"][1:]):
        for h in range(c["kv_heads"]):
            yield slice(a, b), h, slice(h * group, (h + 1) * group)


def _weights(s, rows, h, heads):
    """Softmax weights of every query head of the group (32 bits) and their log-sum-exp."""
    q, k = s["q"][rows, heads].float().transpose(0, 1), s["k"][rows, h].float()
    z = (q @ k.T).mul_(s["scale"])
    n = k.shape[0]
    z.masked_fill_(torch.ones(n, n, dtype=torch.bool, device="cuda").triu_(1), -math.inf)
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(total), (top + total.log())[..., 0], q, k


def _plain_attention(s):
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    for rows, h, heads in _pieces(s):
        p, lse[heads, rows], _, _ = _weights(s, rows, h, heads)
        out[rows, heads] = (p @ s["v"][rows, h].float()).transpose(0, 1).to(out.dtype)
    return {"out": out, "lse": lse}


def _plain_attention_grad(s):
    r = {n: torch.zeros_like(s[n]) for n in ("dq", "dk", "dv")}
    for rows, h, heads in _pieces(s):
        p, _, q, k = _weights(s, rows, h, heads)
        do, v = s["dout"][rows, heads].float().transpose(0, 1), s["v"][rows, h].float()
        r["dv"][rows, h] = (p.transpose(1, 2) @ do).sum(0).to(r["dv"].dtype)
        dp = do @ v.T
        dz = p.mul_(dp.sub_((p * dp).sum(-1, keepdim=True))).mul_(s["scale"])
        r["dq"][rows, heads] = (dz @ k).transpose(0, 1).to(r["dq"].dtype)
        r["dk"][rows, h] = (dz.transpose(1, 2) @ q).sum(0).to(r["dk"].dtype)
    return r


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["grads"]:
        total += t.float().square().sum()
    norm = total.sqrt().float()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0)
    return {"norm": norm, "grads": [(t.float() * factor).to(o.dtype) for t, o in zip(s["grads"], s["outs"])]}


def _workspace(s, nbytes):
    ws = s.get("workspace")
    if ws is None:  # kept with the state, as a program keeps it from call to call
        ws = s["workspace"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
    return ws


def _library(s):
    import paper_2608_00455_b200 as dte

    c, op = s["case"], s["case"]["op"]
    if op == "rope":
        dte.dte_rope(s["q"], s["k"], s["positions"], s["freq"], s["q_out"], s["k_out"], interleaved=c["interleaved"],
                     amplitude=s["amplitude"], inverse=c["inverse"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "attention":
        dte.dte_attention_forward(s["q"], s["k"], s["v"], s["plan"], s["out"], s["lse"], scale=s["scale"])
        return {"out": s["out"], "lse": s["lse"]}
    if op == "attention_grad":
        ws = s.get("workspace")
        if ws is None:
            ws = _workspace(s, dte.dte_attention_backward_workspace_bytes(s["q"].shape[0], c["heads"]))
        dte.dte_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["plan"], s["dq"], s["dk"], s["dv"], ws,
                                   scale=s["scale"])
        return {n: s[n] for n in ("dq", "dk", "dv")}
    ws = s.get("workspace")
    if ws is None:
        ws = _workspace(s, dte.dte_grad_sum_squares_workspace_bytes(len(s["grads"])))
    dte.dte_grad_sum_squares(s["grads"], s["sum_squares"], ws)
    dte.dte_grad_clip(s["grads"], s["sum_squares"], s["max_norm"], s["norm"], s["outs"])
    return {"norm": s["norm"], "grads": s["outs"]}


_PLAIN = {"rope": _plain_rope, "attention": _plain_attention, "attention_grad": _plain_attention_grad, "clip": _plain_clip}


def run(state):
    return _library(state) if own else _PLAIN[state["case"]["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    op = case["op"]
    if op == "rope":
        h = case["heads"] + case["kv_heads"]
        return {"bytes": 2 * case["tokens"] * h * case["head_dim"] * _size(case["dtype"]) + 8 * case["tokens"] + 4 * case["rot"],
                "flops": 3 * case["tokens"] * h * case["rot"]}
    if op == "clip":
        n = sum(a * b for a, b in _shapes(case))
        return {"bytes": n * (_size(case["dtype"]) + _size(case["out"])) + 12, "flops": 3 * n}
    seen = sum(n * (n + 1) // 2 for n in _lengths(case))         # pairs of a query and a key that it sees
    t, hq, hk, d = case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
    if op == "attention":
        return {"bytes": 2 * t * d * (2 * hq + 2 * hk) + 4 * t * hq, "flops": 4 * d * hq * seen}
    return {"bytes": 2 * t * d * (4 * hq + 4 * hk) + 4 * t * hq, "flops": 10 * d * hq * seen}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_rope(case, s):
    # pairs as complex numbers, turned by exp(i angle)
    angle = torch.outer(s["positions"].to(torch.float64), s["freq"])
    turn = torch.polar(torch.full_like(angle, s["amplitude"]), -angle if case["inverse"] else angle)[:, None, :]
    out = {}
    for name in ("q", "k"):
        x = s[name].to(torch.float64)
        head, tail = x[..., :case["rot"]], x[..., case["rot"]:]
        pairs = head.unflatten(-1, (-1, 2)) if case["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        out[name] = torch.cat([z.flatten(-2), tail], -1)
    return out


def _exact_attention(case, s):
    dbl = torch.float64
    grad = case["op"] == "attention_grad"
    rows, hq, d = s["q"].shape
    group = hq // case["kv_heads"]
    names = ("dq", "dk", "dv") if grad else ("out",)
    r = {n: torch.zeros(s[n].shape, dtype=dbl, device="cuda") for n in names}
    if not grad:
        r["lse"] = torch.zeros(hq, rows, dtype=dbl, device="cuda")
    for a, b in zip(s["bounds"][:-1], s["bounds"][1:]):
        for h in range(hq):
            q, k, v = s["q"][a:b, h].to(dbl), s["k"][a:b, h // group].to(dbl), s["v"][a:b, h // group].to(dbl)
            for i in range(0, b - a, 4096):            # blocks of queries, and the keys up to their last one
                j = min(i + 4096, b - a)
                z = torch.mm(q[i:j], k[:j].t()) * s["scale"]
                z += torch.full((j - i, j), -math.inf, dtype=dbl, device="cuda").triu_(i + 1)
                norm = torch.logsumexp(z, 1, keepdim=True)
                p = torch.exp(z - norm)
                if not grad:
                    r["lse"][h, a + i:a + j] = norm[:, 0]
                    r["out"][a + i:a + j, h] = torch.mm(p, v[:j])
                    continue
                do = s["dout"][a + i:a + j, h].to(dbl)
                r["dv"][a:a + j, h // group] += torch.mm(p.t(), do)
                # derivative of the softmax: each weight's gradient less what the row's weights give together
                w = torch.mm(do, v[:j].t())
                w = p * (w - torch.einsum("ij,ij->i", p, w)[:, None]) * s["scale"]
                r["dq"][a + i:a + j, h] = torch.mm(w, k[:j])
                r["dk"][a:a + j, h // group] += torch.mm(w.t(), q[i:j])
    return r


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    if case["op"] != "clip":
        return _exact_attention(case, s)
    norm = torch.stack([torch.linalg.vector_norm(t.to(torch.float64)) for t in s["grads"]]).norm()
    scale = s["max_norm"] / norm if float(norm) > s["max_norm"] else 1.0
    return {"norm": norm, "grads": [t.to(torch.float64) * scale for t in s["grads"]]}
