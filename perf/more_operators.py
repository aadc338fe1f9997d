"""Timed cases of the operators around the LM head on device memory: what teaches an exit head (or a draft model) what the
target model says, and what reports it.

Four operators, in the order in which a step of such a training uses them:

* `score` (`ee_score_tokens`): the target's logits give the log-probabilities of given tokens, the entropy of every row and its
  most likely tokens, which a server reports and which the student learns from;
* `linear` (`ee_linear`, `ee_linear_grad`): the student's products: an exit's adapters, y = act(x W^T + b) + residual, the LM head,
  a single client's rows as well as a prompt's; backward the gradients of inputs, weights and bias;
* `norm` (`ee_norm`, `ee_norm_grad`): the norm in front of the head, with the reduction of the gains' gradient;
* `distill` (`ee_distill`): the divergence of the student's distribution from the teacher's most likely tokens, and its gradient.

Sizes are those of the repository's own configurations (256 and 1024 tokens; width 4096, 11008, 5120; adapters of 384 hidden units in
all; 32000 tokens; prompts of 2041 rows) and generic ones of larger vocabularies.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5


def listed():
    return [
        # one client's round of four drafts on the 7B shape's vocabulary: what its tokens had for a probability, with a few alternatives
        _score("score_round_5x32000", rows=5, vocab=32000, dtype="fp32", top=4, temperature=1.0),
        # a whole prompt's log-probabilities, and the teacher's side of a training step
        _score("score_prompt_2041x32000", rows=2041, vocab=32000, dtype="bf16", top=20, temperature=0.8),
        # a small batch on the repository's smallest model: a call of nothing but latency
        _distill("distill_64x1024", rows=64, vocab=1024, dtype="fp32", top=8, rest=True, grad=True, temperature=1.0),
        # a training step's rows on the 7B shape's vocabulary, loss and gradient
        _distill("distill_4096x32000", rows=4096, vocab=32000, dtype="bf16", top=32, rest=True, grad=True, temperature=2.0),
        # the loss alone, as an evaluation takes it, on a larger and odd vocabulary
        _distill("distill_loss_600x100003", rows=600, vocab=100003, dtype="fp16", top=64, rest=False, grad=False, temperature=1.0),
        # one client's five rows in front of the head: latency
        _norm("norm_5x4096", rows=5, dim=4096, dtype="fp32", out="bf16", center=False, grad=False),
        # a training step's rows, backward with the gradients of gains and biases
        _norm("norm_grad_8191x5120", rows=8191, dim=5120, dtype="bf16", out="bf16", center=True, grad=True),
        # five rows through the LM head: the weights' bytes
        _linear("linear_head_5x4096x32000", rows=5, k=4096, n=32000, dtype="bf16", out="fp32", act="none", bias=False, residual="none", grad=False),
        # a prompt through an exit's adapters, down: few columns
        _linear("linear_down_2041x4096x384", rows=2041, k=4096, n=384, dtype="bf16", out="bf16", act="silu", bias=True, residual="none", grad=False),
        # a prompt through a wide layer with an activation
        _linear("linear_2041x4096x11008", rows=2041, k=4096, n=11008, dtype="bf16", out="bf16", act="silu", bias=True, residual="none", grad=False),
        # backward of the adapters' down projection: few columns, the activation's gradient
        _linear("linear_grad_2041x4096x384", rows=2041, k=4096, n=384, dtype="bf16", out="bf16", act="silu", bias=True, residual="none", grad=True),
        # backward of a wide layer, gradients in fp32
        _linear("linear_grad_2041x4096x11008", rows=2041, k=4096, n=11008, dtype="bf16", out="fp32", act="none", bias=True, residual="none", grad=True),
    ]


def _score(name, **kw):
    return dict(name=name, op="score", pad=0, **kw)


def _distill(name, **kw):
    return dict(name=name, op="distill", pad=0, **kw)


def _norm(name, **kw):
    return dict(name=name, op="norm", pad=0, **kw)


def _linear(name, **kw):
    return dict(name=name, op="linear", pad=0, **kw)


def draw(rng):
    def log_size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def size_within(lo, hi, most):
        return log_size(lo, max(min(hi, most), lo))

    op = rng.choice(["score", "distill", "norm", "linear", "linear"])
    if op in ("score", "distill"):
        vocab = log_size(400, 131072)
        rows = size_within(1, 8192, (2041 if op == "score" else 4096) * 32000 // vocab)
        case = dict(op=op, pad=rng.choice([0, 0, 3]), rows=rows, vocab=vocab, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    top=log_size(1, 64), temperature=rng.choice([1.0, 1.0, 0.7, 2.0]))
        return case if op == "score" else dict(case, rest=rng.random() < 0.5, grad=rng.random() < 0.7)
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "norm":
        dim = log_size(64, 16384)
        dim = dim if rng.random() < 0.3 else -(-dim // 8) * 8
        return dict(op=op, pad=rng.choice([0, 0, 3]), rows=size_within(1, 16384, 8191 * 5120 // dim), dim=dim, dtype=rng.choice([dtype, "fp32"]),
                    out=rng.choice([dtype, "fp32"]), center=rng.random() < 0.5, grad=rng.random() < 0.6)
    k, n = log_size(32, 16384), log_size(32, 16384)
    if rng.random() < 0.7:
        k, n = -(-k // 8) * 8, -(-n // 8) * 8
    rows = size_within(1, 8192, 2041 * 4096 * 11008 // (k * n))
    return dict(op=op, pad=rng.choice([0, 0, 1]), rows=rows, k=k, n=n, dtype=dtype, out=rng.choice([dtype, dtype, "fp32"]), act=rng.choice(["none", "silu", "gelu"]),
                bias=rng.random() < 0.6, residual=rng.choice(["none", dtype, "fp32"]), grad=rng.random() < 0.5)


def work(case):
    op, rows = case["op"], case["rows"]
    size = SIZE[case["dtype"]]
    if op in ("score", "distill"):
        logits, tops = rows * case["vocab"], rows * case["top"] * 8
        moved = logits * size * (2 if op == "distill" and case["grad"] else 1)
        return {"bytes": moved + tops + rows * 12, "flops": 6 * logits}
    out = SIZE[case["out"]]
    if op == "norm":
        n = rows * case["dim"]
        moved = n * (size + out + size) if case["grad"] else n * (size + out)   # x, dy and dx; x and y
        return {"bytes": moved + 12 * case["dim"], "flops": (12 if case["grad"] else 5) * n}
    k, n = case["k"], case["n"]
    x, w, y = rows * k, n * k, rows * n
    if case["grad"]:
        # dy (and the activation's input), x and the weights once; the gradients of inputs, weights and bias
        moved = y * size * (1 if case["act"] == "none" else 2) + (x + w) * size + x * out + w * out + 4 * n
        return {"bytes": moved, "flops": 4 * rows * k * n}
    extra = (SIZE[case["residual"]] if case["residual"] != "none" else 0) + (size if case["act"] != "none" else 0)
    return {"bytes": (x + w) * size + y * (out + extra) + 4 * n * case["bias"], "flops": 2 * rows * k * n}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _generator(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def rows_of(x, dtype, multiple=1):
        """x as a view of rows that are apart from each other, as a slice of a wider array is."""
        width = x.shape[1]
        stride = -(-width // multiple) * multiple + case["pad"] * multiple
        wide = torch.zeros(x.shape[0], stride, dtype=dtype, device="cuda")
        wide[:, :width] = x
        return wide[:, :width]

    op, rows, dtype = case["op"], case["rows"], TYPES[case["dtype"]]
    st = dict(case=case)
    if op in ("score", "distill"):
        V, k = case["vocab"], case["top"]
        # a trained model's logits: one token of a row stands out
        z = 2.0 * normal(rows, V)
        z.scatter_add_(1, torch.randint(V, (rows, 1), generator=g, device="cuda"), math.log(V) + 3.0 + normal(rows, 1))
        st["logits"] = rows_of(z, dtype)
        if op == "score":
            st["tokens"] = torch.randint(V, (rows,), generator=g, device="cuda").int()
            st["logprob"], st["entropy"] = torch.empty(2, rows, device="cuda")
            st["top_ids"] = torch.empty(rows, k, dtype=torch.int32, device="cuda")
            st["top_logprobs"] = torch.empty(rows, k, device="cuda")
            return st
        # the teacher is near its student; its most likely tokens are the training's data
        z = (z + 0.7 * normal(rows, V)) / case["temperature"]
        z -= z.logsumexp(1, keepdim=True)
        values, ids = z.topk(k, dim=1)
        st["ids"], st["logprobs"] = ids.int().contiguous(), values.contiguous()
        st["loss"] = torch.empty(rows, device="cuda")
        if case["grad"]:
            # a mean over the rows, and rows that do not count
            st["d_loss"] = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, 0.0, 1.0 / rows)
            st["d_logits"] = rows_of(torch.empty(rows, V, device="cuda"), dtype)
        return st
    if op == "norm":
        dim = case["dim"]
        st["x"] = rows_of(normal(rows, dim) * (0.5 + torch.rand(rows, 1, generator=g, device="cuda")) + 0.3 * case["center"], dtype)
        st["gain"] = 0.5 + torch.rand(dim, generator=g, device="cuda")
        st["bias"] = 0.1 * normal(dim) if case["center"] else None
        if case["grad"]:
            st["dy"] = rows_of(normal(rows, dim), TYPES[case["out"]])
            st["dx"] = rows_of(torch.empty(rows, dim, device="cuda"), dtype)
            st["d_gain"], st["d_bias"] = torch.empty(2, dim, device="cuda")
        else:
            st["y"] = rows_of(torch.empty(rows, dim, device="cuda"), TYPES[case["out"]])
        return st
    k, n, out = case["k"], case["n"], TYPES[case["out"]]
    st["x"] = rows_of(normal(rows, k), dtype, 8)
    st["weight"] = rows_of(0.02 * normal(n, k), dtype, 8)
    if case["grad"]:
        st["dy"] = rows_of(normal(rows, n), dtype, 8)
        st["pre"] = rows_of(normal(rows, n), dtype, 8) if case["act"] != "none" else None
        st["dx"], st["d_weight"] = rows_of(torch.empty(rows, k, device="cuda"), out, 8), rows_of(torch.empty(n, k, device="cuda"), out, 8)
        st["d_bias"] = torch.empty(n, device="cuda")
        return st
    st["bias"] = 0.02 * normal(n) if case["bias"] else None
    st["residual"] = rows_of(normal(rows, n), TYPES[case["residual"]], 8) if case["residual"] != "none" else None
    st["y"] = rows_of(torch.empty(rows, n, device="cuda"), out, 8)
    st["pre"] = rows_of(torch.empty(rows, n, device="cuda"), dtype, 8) if case["act"] != "none" else None
    return st


# ---------------------------------------------------------------- plain forms

def _plain_score(st):
    z = st["logits"].float()
    rows, V = z.shape
    # an order without ties: the larger logit first, of equal ones the lower token
    bits = (z + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * 2 ** 32 + torch.arange(V - 1, -1, -1, device="cuda")
    ids = V - 1 - (key.topk(st["case"]["top"], dim=1)[0] & 0xFFFFFFFF)
    z = z / st["case"]["temperature"]
    z = z - z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    lse = torch.log(total)
    entropy = lse[:, 0] - (e * z).sum(1) / total[:, 0]
    logprob = (z.gather(1, st["tokens"].long()[:, None]) - lse)[:, 0]
    return {"logprob": logprob, "entropy": entropy, "top_ids": ids.int(), "top_logprobs": z.gather(1, ids) - lse}


def _plain_distill(st):
    """A row's sums and its loss in 64 bits: it is a small difference of large terms, and what the teacher leaves over is one."""
    case, T = st["case"], st["case"]["temperature"]
    z = st["logits"].float()
    top = z.amax(1, keepdim=True)
    q = torch.exp((z - top) / T)
    total = q.sum(1, keepdim=True, dtype=torch.float64)
    ids, log_p = st["ids"].long(), st["logprobs"].double()
    log_q = (z.gather(1, ids).double() - top) / T - torch.log(total)
    p = torch.exp(log_p)
    if case["rest"]:
        pi = (1 - p.sum(1, keepdim=True)).clamp(min=0)
        rho = q.scatter(1, ids, 0.0).sum(1, keepdim=True, dtype=torch.float64) / total
        loss = (p * (log_p - log_q)).sum(1) + (pi * (torch.log(pi.clamp(min=1e-300)) - torch.log(rho)))[:, 0]
        others = (1 - pi / rho).float()
    else:
        share = p.sum(1, keepdim=True)
        log_p, p = log_p - torch.log(share), p / share
        loss = (p * (log_p - log_q)).sum(1)
        others = 1.0
    if not case["grad"]:
        return {"loss": loss.float()}
    weight = st["d_loss"][:, None] / T
    grad = (q * (others / total.float())).scatter(1, ids, (torch.exp(log_q) - p).float()) * weight
    return {"loss": loss.float(), "d_logits": grad.to(st["logits"].dtype)}


def _plain_norm(st):
    case = st["case"]
    x = st["x"].float()
    if case["center"]:
        x = x - x.mean(1, keepdim=True)
    r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    x = x * r
    if not case["grad"]:
        y = x * st["gain"]
        return {"y": (y + st["bias"] if case["center"] else y).to(TYPES[case["out"]])}
    dy = st["dy"].float()
    d = dy * st["gain"]
    dx = d - x * (d * x).mean(1, keepdim=True)
    if case["center"]:
        dx = dx - d.mean(1, keepdim=True)
    return {"dx": (dx * r).to(st["x"].dtype), "d_gain": (dy * x).sum(0), "d_bias": dy.sum(0)}


def _act(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z if act == "none" else 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))


def _act_grad(z, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5


def _plain_linear(st):
    case, out = st["case"], TYPES[st["case"]["out"]]
    x, w = st["x"].float(), st["weight"].float()
    if case["grad"]:
        dz = st["dy"].float()
        if case["act"] != "none":
            dz = dz * _act_grad(st["pre"].float(), case["act"])
        return {"dx": (dz @ w).to(out), "d_weight": (dz.t().contiguous() @ x).to(out), "d_bias": dz.sum(0)}
    z = x @ w.t()
    if case["bias"]:
        z = z + st["bias"]
    y = _act(z, case["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return {"y": y.to(out)} if case["act"] == "none" else {"y": y.to(out), "pre": z.to(st["x"].dtype)}


# ---------------------------------------------------------------- the framework's

def _workspace(st, size):
    if "workspace" not in st:
        st["workspace"] = torch.empty(size(), dtype=torch.uint8, device="cuda")
    return st["workspace"]


def _own(st):
    import paper_2505_21594_amd as ee

    case, stream = st["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "score":
        ws = _workspace(st, lambda: ee.ee_score_workspace(st["logits"], top=case["top"]))
        ee.ee_score_tokens(st["logits"], st["tokens"], logprob=st["logprob"], entropy=st["entropy"], top_ids=st["top_ids"], top_logprobs=st["top_logprobs"],
                           temperature=case["temperature"], workspace=ws, stream=stream)
        return {k: st[k] for k in ("logprob", "entropy", "top_ids", "top_logprobs")}
    if case["op"] == "distill":
        ws = _workspace(st, lambda: ee.ee_distill_workspace(st["logits"], top=case["top"]))
        ee.ee_distill(st["logits"], st["ids"], st["logprobs"], loss=st["loss"], d_loss=st.get("d_loss"), d_logits=st.get("d_logits"), rest=case["rest"],
                      temperature=case["temperature"], workspace=ws, stream=stream)
        return {"loss": st["loss"], "d_logits": st["d_logits"]} if case["grad"] else {"loss": st["loss"]}
    if case["op"] == "norm":
        if not case["grad"]:
            ee.ee_norm(st["x"], st["y"], gain=st["gain"], bias=st["bias"], eps=EPS, center=case["center"], stream=stream)
            return {"y": st["y"]}
        ws = _workspace(st, lambda: ee.ee_norm_grad_workspace(st["x"]))
        ee.ee_norm_grad(st["x"], st["dy"], dx=st["dx"], gain=st["gain"], d_gain=st["d_gain"], d_bias=st["d_bias"], eps=EPS, center=case["center"], workspace=ws, stream=stream)
        return {k: st[k] for k in ("dx", "d_gain", "d_bias")}
    act = {"none": ee.ACT_NONE, "silu": ee.ACT_SILU, "gelu": ee.ACT_GELU}[case["act"]]
    if case["grad"]:
        ws = _workspace(st, lambda: ee.ee_linear_grad_workspace(st["x"], st["weight"], act=act))
        ee.ee_linear_grad(st["x"], st["weight"], st["dy"], pre=st["pre"], act=act, dx=st["dx"], d_weight=st["d_weight"], d_bias=st["d_bias"], workspace=ws, stream=stream)
        return {k: st[k] for k in ("dx", "d_weight", "d_bias")}
    ws = _workspace(st, lambda: ee.ee_linear_workspace(st["x"], st["weight"]))
    ee.ee_linear(st["x"], st["weight"], st["y"], bias=st["bias"], act=act, residual=st["residual"], pre=st["pre"], workspace=ws, stream=stream)
    return {"y": st["y"]} if case["act"] == "none" else {"y": st["y"], "pre": st["pre"]}


def run(state):
    if own:
        return _own(state)
    return {"score": _plain_score, "distill": _plain_distill, "norm": _plain_norm, "linear": _plain_linear}[state["case"]["op"]](state)


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op in ("score", "distill"):
        T, found = case["temperature"], []
        # some rows at a time: 64 bits of them all may not fit
        step = max(1, 2 ** 26 // case["vocab"])
        for at in range(0, case["rows"], step):
            part = slice(at, at + step)
            raw = st["logits"][part].double()
            log_q = torch.log_softmax(raw / T, 1)
            if op == "score":
                best = torch.sort(raw, dim=1, descending=True, stable=True)[1][:, : case["top"]]
                p = torch.softmax(raw / T, 1)
                picked = torch.take_along_dim(log_q, st["tokens"][part].long()[:, None], 1)[:, 0]
                found.append((picked, -torch.special.xlogy(p, p).sum(1), torch.take_along_dim(log_q, best, 1)))
                continue
            ids, log_p = st["ids"][part].long(), st["logprobs"][part].double()
            top = torch.zeros_like(log_q, dtype=torch.bool).scatter_(1, ids, True)
            p = torch.zeros_like(log_q).scatter_(1, ids, log_p.exp())
            gap = torch.take_along_dim(log_q, ids, 1)
            q = log_q.exp()
            if case["rest"]:
                # the tokens that the teacher does not name are one class
                outside = torch.logsumexp(torch.where(top, -math.inf, log_q), 1)
                left = -torch.expm1(torch.logsumexp(log_p, 1)).clamp(max=0)
                loss = (log_p.exp() * (log_p - gap)).sum(1) + torch.special.xlogy(left, left) - torch.where(left > 0, left * outside, 0.0)
                shares = torch.where(top, p, left[:, None] * (log_q - outside[:, None]).exp())
                grad = q - shares
            else:
                log_p = log_p - torch.logsumexp(log_p, 1, keepdim=True)
                loss = (log_p.exp() * (log_p - gap)).sum(1)
                grad = q - p / p.sum(1, keepdim=True)
            found.append((loss, grad * st["d_loss"][part].double()[:, None] / T) if case["grad"] else (loss,))
        found = [torch.cat(x) for x in zip(*found)]
        if op == "score":
            return {"logprob": found[0], "entropy": found[1], "top_ids": None, "top_logprobs": found[2]}
        return {"loss": found[0], "d_logits": found[1]} if case["grad"] else {"loss": found[0]}
    if op == "norm":
        x = st["x"].double()
        if case["grad"]:
            dy, g = st["dy"].double(), st["gain"].double()
            mean = x.mean(1, keepdim=True) if case["center"] else 0.0
            sd = ((x - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt()
            unit = (x - mean) / sd
            # the gradient through the row's standard deviation and mean: the part of dy g that changes neither
            u = dy * g
            along = (u * unit).sum(1, keepdim=True) / case["dim"]
            flat = u.sum(1, keepdim=True) / case["dim"] if case["center"] else 0.0
            return {"dx": (u - flat - unit * along) / sd, "d_gain": torch.einsum("rd,rd->d", dy, unit), "d_bias": dy.sum(0)}
        mean = x.mean(1, keepdim=True) if case["center"] else torch.zeros_like(x[:, :1])
        y = (x - mean) / ((x - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt() * st["gain"].double()
        return {"y": y + st["bias"].double() if case["center"] else y}
    x, w = st["x"].double(), st["weight"].double()
    if case["grad"]:
        dz = st["dy"].double()
        if case["act"] == "silu":
            z = st["pre"].double()
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        elif case["act"] == "gelu":
            z = st["pre"].double()
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        return {"dx": torch.mm(dz, w), "d_weight": torch.mm(dz.t(), x), "d_bias": dz.sum(0)}
    z = torch.mm(x, w.t())
    if st["bias"] is not None:
        z = z + st["bias"].double()
    y = {"none": lambda: z, "silu": lambda: z * torch.sigmoid(z), "gelu": lambda: z * torch.special.ndtr(z)}[case["act"]]()
    if st["residual"] is not None:
        y = y + st["residual"].double()
    return {"y": y} if case["act"] == "none" else {"y": y, "pre": z}
