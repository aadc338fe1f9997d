"""Timed cases of the operators on device memory: the steps of a decoder layer's attention and of a
round's verification, as a server calls them that runs a model of its own around the library's paged cache.

Three operators, in the order in which such a server uses them:

* `append` (`ee_kv_append`): the new rows' queries and keys are normalised per head where the model does that,
  rotated to their positions, and the keys and values go into the sequences' pages;
* `attend` (`ee_attend`): the rows' queries attend to the pages, the pages that sequences have in common (a
  system prompt, an image) being read once for all of them;
* `accept` (`ee_accept_drafts`): the rows' logits decide how many drafted tokens of every sequence stay and which
  token follows, from given random numbers.

Sizes are those of the repository's own configurations (4 heads of 64 and 1024 tokens; 32 and 40 heads of 128 and 32000
tokens; 576 image rows; prompts of 2041) and generic ones of shared key heads and larger vocabularies.
A list of lengths is written "a,b,c", or "n*lo-hi": n lengths from lo to hi, spread over their logarithm.
"""
import math

import torch

own = False

PAGE = 16
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


def listed():
    return [
        # the repository's smallest model: one client's five rows behind 64 positions, as its session caches them
        _append("append_tiny_5", heads=4, kv_heads=4, dim=64, terms=2, dtype="fp32", rows="5", start="64", norm=False, pairs=False),
        # eight clients' rounds of five rows on the 7B shape, their images and questions cached already
        _append("append_b8_rounds", heads=32, kv_heads=32, dim=128, terms=2, dtype="fp32", rows="8*5-5", start="8*640-667", norm=True, pairs=True),
        # a mixed batch: single tokens, rounds and prompts of many clients in one call, shared key heads, per-head norms
        _append("append_mixed_b24", heads=32, kv_heads=8, dim=128, terms=1, dtype="bf16", rows="24*1-300", start="24*0-1100", norm=True, pairs=False),
        # a long prompt
        _append("append_prompt_2041", heads=32, kv_heads=32, dim=128, terms=1, dtype="bf16", rows="2041", start="0", norm=False, pairs=False),
        # the smallest model's round: a call of nothing but latency
        _attend("attend_tiny_5", heads=4, kv_heads=4, dim=64, terms=2, dtype="fp32", rows="5", own="69", shared="0", members="1"),
        # eight clients that sent questions about one image: 576 positions in common
        _attend("attend_b8_image", heads=32, kv_heads=32, dim=128, terms=2, dtype="fp32", rows="8*5-5", own="8*64-90", shared="576", members="8"),
        # single tokens of 32 clients of one application behind its long instructions
        _attend("attend_b32_instructions", heads=32, kv_heads=8, dim=128, terms=1, dtype="bf16", rows="32*1-1", own="32*40-1500", shared="6000", members="32"),
        # two applications and a client of neither, rounds of various lengths, head size 64
        _attend("attend_two_groups", heads=12, kv_heads=4, dim=64, terms=1, dtype="fp16", rows="13*1-16", own="13*16-2000", shared="1000,333,0", members="7,5,1"),
        # one client far into a long document: a single row, all of the chip on one cache
        _attend("attend_single_60k", heads=32, kv_heads=8, dim=128, terms=1, dtype="bf16", rows="1", own="60001", shared="0", members="1"),
        # a prompt's rows, the matrix cores' case
        _attend("attend_prompt_2041", heads=32, kv_heads=32, dim=128, terms=1, dtype="bf16", rows="2041", own="2041", shared="0", members="1"),
        # one client's round of four drafts on the 7B shape's vocabulary
        _accept("accept_g4_32000", vocab=32000, dtype="fp32", rows="5", greedy=False),
        # many clients' rounds of various lengths on a larger vocabulary
        _accept("accept_b24_100k", vocab=100003, dtype="bf16", rows="24*2-9", greedy=False),
    ]


def _append(name, **kw):
    return dict(name=name, op="append", pad=0, **kw)


def _attend(name, **kw):
    return dict(name=name, op="attend", pad=0, **kw)


def _accept(name, **kw):
    return dict(name=name, op="accept", pad=0, **kw)


def draw(rng):
    def log_size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def lengths(n, lo, hi):
        a, b = sorted((log_size(max(lo, 1), hi), log_size(max(lo, 1), hi)))
        return "%d*%d-%d" % (n, max(a - 1, 0) if lo == 0 else a, b)

    op = rng.choice(["append", "append", "attend", "attend", "attend", "accept"])
    if op == "accept":
        n = log_size(1, 32)
        return dict(op=op, pad=rng.choice([0, 0, 3]), vocab=log_size(1000, 131072), dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                    rows=lengths(n, 1, 16), greedy=rng.random() < 0.2)
    dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 10, 32])
    group = rng.choice([1, 1, 2, 3, 4, 8]) if kv_heads < 32 else 1
    terms = rng.choice([1, 1, 2])
    dtype = "fp32" if terms == 2 else rng.choice(["bf16", "bf16", "fp16", "fp32"])
    base = dict(op=op, pad=rng.choice([0, 0, 5]), heads=kv_heads * group, kv_heads=kv_heads, dim=dim, terms=terms, dtype=dtype)
    if op == "append":
        n = log_size(1, 32)
        return dict(base, rows=lengths(n, 1, 2041 // n + 1), start=lengths(n, 0, 1500), norm=rng.random() < 0.6, pairs=rng.random() < 0.4)
    n = log_size(1, 32)
    long_rows = rng.random() < 0.25
    most = 60000 * 8 * 128 // (kv_heads * dim * terms)  # positions, by the cache's bytes
    rows = lengths(n, 1, 38400 // (n * max(kv_heads * group, 32)) + 1 if long_rows else 16)
    members, left = [], n
    while left:
        members.append(rng.randint(1, left) if len(members) < 3 else left)
        left -= members[-1]
    shared = [log_size(16, min(8000, most // 10) if not long_rows else 500) if m > 1 and rng.random() < 0.8 else 0 for m in members]
    return dict(base, rows=rows, own=lengths(n, 2, most * 2 // 3 // n + 2 if not long_rows else 1500 // n + 20), shared=",".join(map(str, shared)), members=",".join(map(str, members)))


# ---------------------------------------------------------------- sizes

def _lengths(text):
    if "*" not in text:
        return [int(x) for x in text.split(",")]
    n, span = text.split("*")
    lo, hi = (int(x) for x in span.split("-"))
    n = int(n)
    low = max(lo, 1)
    out = [int(round(low * (hi / low) ** (((i * 7919) % n) / max(n - 1, 1)))) for i in range(n)]
    return [lo if x == low else x for x in out]


def _starts(rows):
    out = [0]
    for r in rows:
        out.append(out[-1] + r)
    return out


def _layout(case):
    """Rows of every sequence, cached positions (this call's included), positions in common with its group."""
    rows = _lengths(case["rows"])
    if case["op"] == "append":
        return rows, [s + r for s, r in zip(_lengths(case["start"]), rows)], [0] * len(rows)
    members, shared = _lengths(case["members"]), [s // PAGE * PAGE for s in _lengths(case["shared"])]
    common = [s for s, m in zip(shared, members) for _ in range(m)]
    lens = [c + max(o, r) for c, o, r in zip(common, _lengths(case["own"]), rows)]
    return rows, lens, common


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
    if case["op"] == "accept":
        rows = _lengths(case["rows"])
        V = case["vocab"]
        # logits once, the draft distribution of the row that ends the round; a few operations a logit
        drafts = 0 if case["greedy"] else len(rows) * V * 4
        return {"bytes": sum(rows) * V * size + drafts, "flops": 4 * sum(rows) * V}
    rows, lens, common = _layout(case)
    H, Hk, hd, terms = case["heads"], case["kv_heads"], case["dim"], case["terms"]
    T = sum(rows)
    if case["op"] == "append":
        return {"bytes": T * hd * ((2 * H + 2 * Hk) * size + 2 * Hk * terms * 2) + T * hd * 4, "flops": T * (H + Hk) * hd * 8}
    read = sum(n - c for n, c in zip(lens, common))
    at = 0
    for m in _lengths(case["members"]):
        read += common[at]
        at += m
    seen = sum(r * (n - r) + r * (r + 1) // 2 for r, n in zip(rows, lens))
    return {"bytes": read * Hk * hd * terms * 2 * 2 + 2 * T * H * hd * size, "flops": 4 * seen * H * hd}


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _split(x, terms):
    """x as `terms` bf16 terms, on a new axis in front of the last one."""
    hi = x.bfloat16()
    return torch.stack([hi, (x - hi.float()).bfloat16()], dim=-2) if terms == 2 else hi.unsqueeze(-2)


def prepare(case, seed):
    g = _generator(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    dtype = TYPES[case["dtype"]]
    rows = _lengths(case["rows"])
    T, n = sum(rows), len(rows)
    st = dict(case=case, T=T, rows=rows, max_rows=max(rows), row_start=_int(_starts(rows)))
    if case["op"] == "accept":
        V = case["vocab"]
        cap = T + case["pad"]
        # a trained model's logits: one token of a row stands out, the draft model's are near them
        z = 2.0 * normal(cap, V)
        favourite = torch.randint(V, (cap, 1), generator=g, device="cuda")
        z.scatter_add_(1, favourite, math.log(V) + 3.0 + normal(cap, 1))
        st["logits"] = z.to(dtype)
        temperature = torch.full((n,), 0.0, device="cuda") if case["greedy"] else 0.6 + 0.6 * torch.rand(n, generator=g, device="cuda")
        seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(rows, device="cuda"), output_size=T)
        per_row = torch.ones(cap, 1, device="cuda")
        per_row[:T, 0] = temperature[seq].clamp(min=0.5)
        probs = torch.softmax((z + 0.5 * normal(cap, V)) / per_row, dim=1)
        # a draft is drawn from its distribution; a greedy client sends its most likely token
        st["drafts"] = (probs.argmax(1) if case["greedy"] else (probs / torch.empty_like(probs).exponential_(generator=g)).argmax(1)).int()
        st["draft_probs"] = None if case["greedy"] else probs
        st["u"], st["v"] = (torch.rand(cap, generator=g, device="cuda") for _ in range(2))
        st["temperature"] = temperature
        st["accept_len"], st["next_token"] = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        return st
    rows, lens, common = _layout(case)
    H, Hk, hd, terms = case["heads"], case["kv_heads"], case["dim"], case["terms"]
    st.update(kv_len=_int(lens), max_kv=max(lens))
    # a page table as a server's allocator leaves it: pages in no order, a group's common ones the same
    pages = [-(-x // PAGE) for x in lens]
    table, used, at, groups = [], 0, 0, [0]
    members = _lengths(case["members"]) if case["op"] == "attend" else [1] * n
    for m in members:
        shared = list(range(used, used + common[at] // PAGE))
        used += len(shared)
        for s in range(at, at + m):
            mine = list(range(used, used + pages[s] - len(shared)))
            used += len(mine)
            table.append(shared + mine)
        at += m
        groups.append(at)
    stride = max(pages)
    order = torch.randperm(used, generator=g, device="cuda").int()
    padded = torch.tensor([t + [0] * (stride - len(t)) for t in table], device="cuda")
    st["page_table"] = order[padded].contiguous()
    cap = T + case["pad"]
    if case["op"] == "append":
        # one buffer of a row's queries, keys and values, as one projection leaves them
        qkv = (1.25 * normal(cap, H + 2 * Hk, hd)).to(dtype)
        st["q"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        st["q_out"] = torch.zeros(cap, H, hd, dtype=dtype, device="cuda")
        st["q_gain"], st["k_gain"] = ((0.5 + torch.rand(hd, generator=g, device="cuda")) if case["norm"] else None for _ in range(2))
        angle = torch.arange(max(lens), device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, hd, 2, device="cuda", dtype=torch.float64) / hd)
        st["rope"] = torch.stack([angle.cos(), angle.sin()], dim=-1).float()
        st["k_pool"] = torch.zeros(used, Hk, PAGE, terms, hd, dtype=torch.bfloat16, device="cuda")
        st["v_pool"] = torch.zeros(used, Hk, terms, hd, PAGE, dtype=torch.bfloat16, device="cuda")
        return st
    st.update(group_start=_int(groups), group_pages=_int([common[i] // PAGE for i in groups[:-1]]), max_shared=max(common))
    st["q"] = normal(cap, H, hd).to(dtype)
    st["out"] = torch.zeros(cap, H, hd, dtype=dtype, device="cuda")
    k = _split(normal(used, Hk, PAGE, hd), terms)
    st["k_pool"] = k.contiguous()
    v = _split(normal(used, Hk, PAGE, hd), terms)
    st["v_pool"] = v.permute(0, 1, 3, 4, 2).contiguous()
    return st


# ---------------------------------------------------------------- plain forms

def _rows_of(st):
    """Sequence and position of every row in use."""
    r = torch.arange(st["T"], device="cuda")
    seq = torch.searchsorted(st["row_start"][1:].contiguous(), r, right=True)
    return r, seq, st["kv_len"].long()[seq] - st["row_start"].long()[seq + 1] + r


def _rotate(x, cs, pairs):
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if pairs:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * c - b * s, b * c + a * s], dim=-1)


def _plain_append(st):
    case, T = st["case"], st["T"]
    r, seq, pos = _rows_of(st)
    cs = st["rope"][pos]

    def normed(x, gain):
        x = x[:T].float()
        if gain is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
        return _rotate(x, cs, case["pairs"])

    st["q_out"][:T] = normed(st["q"], st["q_gain"]).to(st["q_out"].dtype)
    page, slot = st["page_table"][seq, pos // PAGE].long(), pos % PAGE
    st["k_pool"][page, :, slot] = _split(normed(st["k"], st["k_gain"]), case["terms"])
    st["v_pool"][page, :, :, :, slot] = _split(st["v"][:T].float(), case["terms"])


def _appended(st):
    """The updated cache; of two-term records the rows' values, hi + lo, which is what they stand for."""
    if st["case"]["terms"] == 1:
        return {"q": st["q_out"], "k": st["k_pool"], "v": st["v_pool"]}
    page, slot = st.get("where") or _where(st)
    return {"q": st["q_out"], "k": st["k_pool"][page, :, slot].float().sum(2), "v": st["v_pool"][page, :, :, :, slot].float().sum(2)}


def _where(st):
    r, seq, pos = _rows_of(st)
    st["where"] = st["page_table"][seq, pos // PAGE].long(), pos % PAGE
    return st["where"]


def _plain_attend(st):
    case, T = st["case"], st["T"]
    H, Hk, hd = case["heads"], case["kv_heads"], case["dim"]
    G, M = H // Hk, st["max_rows"]
    table, lens, starts = st["page_table"].long(), st["kv_len"].long(), st["row_start"].long()
    n, P = table.shape
    K = st["k_pool"][table].float().sum(4).transpose(1, 2).reshape(n, Hk, P * PAGE, hd)
    V = st["v_pool"][table].float().sum(3).permute(0, 2, 1, 4, 3).reshape(n, Hk, P * PAGE, hd)
    here = torch.arange(P * PAGE, device="cuda")
    V = torch.where((here < lens[:, None])[:, None, :, None], V, 0.0)
    i = torch.arange(M, device="cuda")
    count = starts[1:] - starts[:-1]
    q = st["q"][:T].float()[(starts[:-1, None] + i).clamp(max=T - 1)]
    q = q.view(n, M, Hk, G, hd).permute(0, 2, 1, 3, 4).reshape(n, Hk, M * G, hd)
    S = torch.matmul(q, K.transpose(-1, -2).contiguous()) * hd ** -0.5
    last = lens[:, None] - count[:, None] + i
    seen = (here <= last[:, :, None]).repeat_interleave(G, 1)[:, None]
    S = S.masked_fill(~seen, -math.inf)
    S = torch.exp(S - S.amax(-1, keepdim=True))
    O = torch.matmul(S, V) / S.sum(-1, keepdim=True)
    r, seq, _ = _rows_of(st)
    O = O.view(n, Hk, M, G, hd)[seq, :, r - starts[seq]]
    st["out"][:T] = O.reshape(T, H, hd).to(st["out"].dtype)
    return {"out": st["out"]}


def _plain_accept(st):
    """In 64 bits: a draw is decided by sums over the vocabulary next to a border."""
    case, T = st["case"], st["T"]
    starts = st["row_start"].long()
    r = torch.arange(T, device="cuda")
    seq = torch.searchsorted(starts[1:].contiguous(), r, right=True)
    z = st["logits"][:T].double()
    draft = st["drafts"][:T].long()
    if case["greedy"]:
        best = z.argmax(1)
        kept = best == draft
    else:
        z = z - z.amax(1, keepdim=True)
        q = torch.exp(z / st["temperature"].double()[seq][:, None])
        q = q / q.sum(1, keepdim=True)
        p = st["draft_probs"][:T]
        kept = st["u"][:T].double() * p[r, draft].double() < q[r, draft]
    kept = kept & (r < starts[seq + 1] - 1)
    # drafts kept before the first that is not: rows whose sequence has lost none up to there
    lost = torch.cumsum((~kept).long(), 0)
    before = torch.cat([lost.new_zeros(1), lost])[starts[seq]]
    st["accept_len"].zero_().scatter_add_(0, seq, (lost == before).int())
    end = starts[:-1] + st["accept_len"]
    if case["greedy"]:
        st["next_token"].copy_(best[end])
    else:
        w = torch.where((end < starts[1:] - 1)[:, None], (q[end] - p[end].double()).clamp(min=0), q[end])
        w = torch.where(w.sum(1, keepdim=True) > 0, w, q[end])
        c = torch.cumsum(w, 1)
        st["next_token"].copy_((c <= st["v"][end].double()[:, None] * c[:, -1:]).sum(1))
    return {"accept_len": st["accept_len"], "next_token": st["next_token"]}


# ---------------------------------------------------------------- the framework's

def _own(st):
    import paper_2505_21594_amd as ee

    case, stream = st["case"], torch.cuda.current_stream().cuda_stream
    if case["op"] == "accept":
        if "workspace" not in st:
            st["workspace"] = torch.empty(ee.ee_accept_workspace(st["logits"], st["row_start"]), dtype=torch.uint8, device="cuda")
        ee.ee_accept_drafts(st["logits"], st["row_start"], st["drafts"], st["draft_probs"], st["u"], st["v"], st["temperature"],
                            st["accept_len"], st["next_token"], workspace=st["workspace"], stream=stream)
        return {"accept_len": st["accept_len"], "next_token": st["next_token"]}
    if "cache" not in st:
        st["cache"] = ee.PagedCache(st["k_pool"], st["v_pool"], st["page_table"])
    if case["op"] == "append":
        ee.ee_kv_append(st["cache"], st["row_start"], st["kv_len"], st["q"], st["k"], st["v"], st["q_out"], q_gain=st["q_gain"], k_gain=st["k_gain"],
                        eps=EPS, rope=st["rope"], rope_pairs=case["pairs"], stream=stream)
        return _appended(st)
    groups = dict(group_start=st["group_start"], group_pages=st["group_pages"], max_shared=st["max_shared"]) if st["max_shared"] else {}
    if "workspace" not in st:
        size = ee.ee_attend_workspace(st["cache"], st["row_start"], st["q"], max_kv=st["max_kv"], **groups)
        st["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    ee.ee_attend(st["cache"], st["row_start"], st["kv_len"], st["q"], st["out"], scale=case["dim"] ** -0.5, max_kv=st["max_kv"],
                 workspace=st["workspace"], stream=stream, **groups)
    return {"out": st["out"]}


def run(state):
    if own:
        return _own(state)
    if state["case"]["op"] == "append":
        _plain_append(state)
        return _appended(state)
    return _plain_attend(state) if state["case"]["op"] == "attend" else _plain_accept(state)


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    rows = _lengths(case["rows"])
    starts = _starts(rows)
    if case["op"] == "accept":
        return None  # whole numbers
    rows, lens, _ = _layout(case)
    H, Hk, hd, terms = case["heads"], case["kv_heads"], case["dim"], case["terms"]
    table = st["page_table"].tolist()
    if case["op"] == "append":
        q_out = st["q_out"].double()
        slots_k, slots_v = (torch.zeros(st["k_pool"].shape[0] * PAGE, Hk, hd, dtype=torch.float64, device="cuda") for _ in range(2))
        taken = []
        for s, count in enumerate(rows):
            for_rows = slice(starts[s], starts[s] + count)
            p = torch.arange(lens[s] - count, lens[s], device="cuda")
            # the rotation multiplies the complex number of a pair by that of its angle, as the table has it
            turn = torch.view_as_complex(st["rope"][p].double())[:, None]

            def turned(x, gain):
                x = x[for_rows].double()
                if gain is not None:
                    x = x / (x.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt() * gain.double()
                if case["pairs"]:
                    return torch.view_as_real(torch.view_as_complex(x.reshape(count, -1, hd // 2, 2).contiguous()) * turn).reshape(x.shape)
                y = torch.complex(x[..., : hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * turn
                return torch.cat([y.real, y.imag], -1)

            q_out[for_rows] = turned(st["q"], st["q_gain"])
            at = [table[s][x // PAGE] * PAGE + x % PAGE for x in range(lens[s] - count, lens[s])]
            taken += at
            slots_k[at] = turned(st["k"], st["k_gain"])
            slots_v[at] = st["v"][for_rows].double()
        if terms == 2:
            return {"q": q_out, "k": slots_k[taken], "v": slots_v[taken]}
        return {"q": q_out, "k": slots_k.view(-1, PAGE, Hk, hd).transpose(1, 2).unsqueeze(3).contiguous(),
                "v": slots_v.view(-1, PAGE, Hk, hd).permute(0, 2, 3, 1).unsqueeze(2).contiguous()}
    if work(case)["flops"] > 2e11:
        return None
    out = st["out"].double()
    for s, count in enumerate(rows):
        own_pages = table[s][: -(-lens[s] // PAGE)]
        for h in range(Hk):
            K = st["k_pool"][own_pages, h].double().sum(2).reshape(-1, hd)[: lens[s]]
            V = st["v_pool"][own_pages, h].double().sum(1).transpose(1, 2).reshape(-1, hd)[: lens[s]]
            heads = slice(h * (H // Hk), (h + 1) * (H // Hk))
            S = torch.tensordot(st["q"][starts[s]: starts[s + 1], heads].double(), K, dims=([2], [1])) / math.sqrt(hd)
            p = torch.arange(lens[s], device="cuda")
            behind = p[None, None, :] > (lens[s] - count + torch.arange(count, device="cuda"))[:, None, None]
            S[behind.expand_as(S)] = -math.inf
            out[starts[s]: starts[s + 1], heads] = torch.tensordot(torch.softmax(S, -1), V, dims=([2], [0]))
    return {"out": out}
