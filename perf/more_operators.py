"""Performance cases of exact rows before their compression: the attention of a
prompt, the pages that rows live in, and the attention of a step over them.

Kinds of cases, each a pass through one operator (or the pair that is always
used together):

* ``prompt`` - causal attention of the tokens of packed prompts, or of the next
               tokens of sequences that hold keys already (``prompt_attn``).
* ``pages``  - one layer's rows written into the pages of their sequences, in
               FP8 with an exponent a row where the cache holds FP8, and rows of
               the same sequences read back (``page_write``, then ``page_read``).
* ``paged``  - one decode step that attends over paged rows (``paged_attn``).

Steps run their layers in the order even, then odd.
"""
import math
import random

import torch

own = False

MOST = {"prompt": 32 * 128 * 32768 * 32768 // 2, "pages": 8 * 128 * 16384, "paged": 8 * 8 * 128 * 131072}

# The 8B shape: 32 query heads on 8 KV heads of 128 channels.  Steps take fewer
# layers than the model has, a pipeline stage's share.
M8B = dict(kv=8, group=4, d=128, dtype="bf16")
PROMPT = dict(M8B, kind="prompt", batch=1, past=0, packed=True)
PAGES = dict(M8B, kind="pages", page=64, batch=1)
STEP = dict(M8B, kind="paged", page=64, layers=8, batch=1, graph=False)


def listed():
    return [
        # a short prompt of a small fp32 model: the smallest call, bound by its launch
        dict(PROMPT, name="prompt_f32_301", kv=4, group=2, d=64, dtype="f32", tmin=301, tmax=301),
        # an ordinary long prompt, odd length
        dict(PROMPT, name="prompt_8b_8k", tmin=8191, tmax=8191),
        # a server's batch of prompts of unlike lengths, packed
        dict(PROMPT, name="prompt_8b_packed24", batch=24, tmin=1, tmax=2000),
        # the next tokens of a long prompt taken in pieces: few rows, many keys, eight query heads to a KV head
        dict(PROMPT, name="prompt_70b_chunk_33k", group=8, tmin=250, tmax=250, past=32768, packed=False),
        # the benchmark's prompt
        dict(PROMPT, name="prompt_8b_32k", tmin=32768, tmax=32768),
        # the new rows of a busy server's step, every sequence at its own position, FP8
        dict(PAGES, name="pages_step_b48_fp8", dtype="bf16_e4m3", batch=48, tokens=48, past=4096),
        # a prompt's rows, FP8, odd length
        dict(PAGES, name="pages_prompt_8k_fp8", dtype="bf16_e4m3", tokens=8191, past=0),
        # a short prompt of a small fp32 model, small pages
        dict(PAGES, name="pages_f32_1001", kv=4, group=2, d=64, dtype="f32", page=16, tokens=1001, past=0),
        # a few conversations of a small fp32 model, captured in a graph as a server does
        dict(STEP, name="paged_f32_1001_b4", layers=2, kv=4, group=2, d=64, dtype="f32", page=16, batch=4, tmin=1, tmax=1001, graph=True),
        # long-context step of one sequence, FP8
        dict(STEP, name="paged_8b_32k_fp8", layers=16, dtype="bf16_e4m3", tmin=32768, tmax=32768, graph=True),
        # a busy server, sequences of unlike lengths, small pages
        dict(STEP, name="paged_8b_b64", batch=64, page=16, tmin=100, tmax=8000),
        # the longest context, eight query heads to a KV head, large pages
        dict(STEP, name="paged_70b_131k", group=8, page=256, tmin=131072, tmax=131072, graph=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "pages", "paged", "paged"])
    c = dict(kind=kind, kv=rng.choice([1, 2, 4, 8, 8]), group=rng.choice([1, 2, 4, 4, 8]), d=rng.choice([64, 128, 128]),
             dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    slow = 8 if c["dtype"] == "f32" else 1
    if kind == "prompt":
        c["batch"] = rng.choice([1, 1, 2, 7, 24])
        c["packed"] = rng.random() < 0.6
        c["past"] = 0 if c["packed"] else rng.choice([0, _log_int(rng, 1, 32768)])
        pairs = MOST[kind] // slow // (c["kv"] * c["group"] * c["d"] * c["batch"])
        most = min(32768, int(math.sqrt(c["past"] ** 2 + pairs)) - c["past"])      # n (past + n / 2) <= pairs, with room
        c["tmax"] = _log_int(rng, 1, max(1, most))
        c["tmin"] = rng.choice([c["tmax"], max(1, c["tmax"] // 8)])
        return c
    c["dtype"] = rng.choice([c["dtype"], "bf16_e4m3"])
    c["page"] = rng.choice([16, 32, 64, 128, 256])
    if kind == "pages":
        c["tokens"] = _log_int(rng, 1, MOST[kind] // slow // (c["kv"] * c["d"]))
        c["batch"] = rng.choice([1, c["tokens"] if c["tokens"] <= 256 else 1])
        c["past"] = rng.randint(0, 3000)
        return c
    c.update(layers=rng.choice([2, 4, 8]), batch=rng.choice([1, 1, 2, 5, 16, 64]), graph=rng.random() < 0.5)
    room = MOST[kind] // slow // (c["layers"] * c["kv"] * c["d"] * c["batch"])
    c["tmax"] = _log_int(rng, 1, min(131072, room))
    c["tmin"] = rng.choice([c["tmax"], max(1, c["tmax"] // 8)])
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed, *tags):
    return torch.Generator("cuda").manual_seed(random.Random("%d %s" % (seed, tags)).getrandbits(62))


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _bytes(t):
    return torch.empty(0, dtype=t).element_size()


def _rand(c, seed, tag, *shape):
    return torch.randn(*shape, generator=_gen(seed, tag), device="cuda").to(_type(c))


def _rows(c, seed, tag, *shape):
    """Key or value rows [..][d]: a few channels are larger than the others, as a model's are, and rows differ in size."""
    g = _gen(seed, tag)
    x = torch.randn(*shape, generator=g, device="cuda")
    x[..., torch.randint(c["d"], (3,), generator=g, device="cuda")] *= 6
    return (x * (0.5 + torch.rand(*shape[:-1], 1, generator=g, device="cuda"))).to(_type(c))


def _scale(c):
    return 1.0 / math.sqrt(c["d"])


def _lengths(c):
    """Lengths over tmin .. tmax, the longest among them: of a case the same ones, in an order that the seed gives."""
    r = random.Random("lengths %d %d %d" % (c["batch"], c["tmin"], c["tmax"]))
    return [r.randint(c["tmin"], c["tmax"]) for _ in range(c["batch"] - 1)] + [c["tmax"]]


def _lens(c, seed):
    lens = _lengths(c)
    random.Random("lens %d" % seed).shuffle(lens)
    return lens


def _table(seed, pages):
    """Page numbers [batch][most] of sequences of so many pages each, scattered over the pool; -1 behind the last."""
    n = sum(pages)
    order = torch.randperm(n, generator=_gen(seed, "table"), device="cuda").to(torch.int32)
    table = torch.full((len(pages), max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, m in enumerate(pages):
        table[s, :m] = order[at:at + m]
        at += m
    return table, n


def prepare(case, seed):
    c = case
    st = dict(case=c)
    kv, hq, d = c["kv"], c["kv"] * c["group"], c["d"]
    i32 = dict(dtype=torch.int32, device="cuda")
    if c["kind"] == "prompt":
        lens = _lens(c, seed)
        n = sum(lens)
        starts = [sum(lens[:s]) for s in range(len(lens) + 1)]
        st.update(lens=lens, starts=starts)
        st["q"] = _rand(c, seed, "q", n, hq, d) * 1.5
        shape = (1, kv, n, d) if c["packed"] else (c["batch"], kv, c["past"] + c["tmax"] + 5, d)
        st["k"], st["v"] = _rows(c, seed, "k", *shape), _rows(c, seed, "v", *shape)
        st["out"] = torch.empty_like(st["q"])
        st["q_starts"] = torch.tensor(starts, **i32)
        st["k_lens"] = torch.tensor([c["past"] + m for m in lens], **i32)
        st["k_starts"] = st["q_starts"][:-1].clone() if c["packed"] else None
    elif c["kind"] == "pages":
        n, r = c["tokens"], random.Random("rows %d" % seed)
        many = c["batch"] > 1
        past = [r.randint(0, c["past"]) for _ in range(c["batch"])]
        new = 1 if many else n
        st["table"], st["n_pages"] = _table(seed, [-(-(p + new) // c["page"]) for p in past])
        # rows as a projection leaves them, keys and values of all heads side by side
        st["kv"] = _rows(c, seed, "kv", n, 2 * kv, d)
        st["seqs"] = torch.arange(n, **i32) if many else torch.zeros(n, **i32)
        st["rows"] = torch.tensor(past, **i32) if many else torch.arange(n, **i32) + past[0]
        st["k_out"], st["v_out"] = (torch.empty(kv, n, d, dtype=_type(c), device="cuda") for _ in range(2))
        st["pools"] = _pools(c, seed, 0, st["n_pages"])
    else:
        lens = _lens(c, seed)
        st["table"], st["n_pages"] = _table(seed, [-(-T // c["page"]) for T in lens])
        st["lens"] = torch.tensor(lens, **i32)
        st["lens_host"] = lens
        st["layers"] = [_pools(c, seed, l, st["n_pages"]) for l in range(c["layers"])]
        st["q"] = _rand(c, seed, "q", c["layers"], c["batch"], hq, d) * 1.5
        st["out"] = torch.empty_like(st["q"])
    if own:
        _handles(st)
    return st


def _power(e):
    """2^(e - 127) in fp32, exactly, for whole numbers 1 <= e <= 254."""
    return (e.int() << 23).view(torch.float32)


def _quantised(x):
    """Rows [..][d] as E4M3 codes and the exponent of each row: the least e with max |x| <= 448 2^e, held as e + 127."""
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1))                                 # max = m 2^e, 1/2 <= m < 1, 448 = 7/8 2^9
    e = torch.where(m == 0, -127, e - 9 + (m > 0.875).to(e.dtype)).clamp(-126, 127)
    return (x * _power(127 - e).unsqueeze(-1)).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _pools(c, seed, layer, n_pages):
    """A layer's pages as sequences before left them: K and V [pages][kv][page][d], and exponents of FP8 rows."""
    shape, st = (n_pages, c["kv"], c["page"], c["d"]), {}
    for t in "kv":
        x = _rows(c, seed, ("pool", layer, t), *shape)
        st[t], st[t + "_exp"] = _quantised(x) if c["dtype"] == "bf16_e4m3" else (x, None)
    return st


def _handles(st):
    """What a program of this framework keeps between calls: descriptors, workspaces, a captured step."""
    from paper_2607_06519_amd import binding as B
    c = st["case"]
    hq = c["kv"] * c["group"]
    st["B"] = B
    dims = st["dims"] = B.dims(c.get("layers", 2), c["kv"], hq, c["d"], 0, c["dtype"])
    if c["kind"] == "prompt":
        n = B.prompt_attn_workspace(dims, st["q"].shape[0], c["batch"], st["k"].shape[2])
        st["ws"] = torch.empty(n // 4 + 64, dtype=torch.float32, device="cuda")
        return
    if c["kind"] == "pages":
        p = st["pools"]
        st["desc"] = B.pages(dims, p["k"], p["v"], st["table"], p["k_exp"], p["v_exp"])
        return
    st["desc"] = [B.pages(dims, p["k"], p["v"], st["table"], p["k_exp"], p["v_exp"]) for p in st["layers"]]
    st["most"] = max(st["lens_host"])
    n = B.paged_attn_workspace(dims, c["batch"], st["most"])
    st["ws"] = torch.empty(n // 4 + 64, dtype=torch.float32, device="cuda")
    if c["graph"]:
        _own_step(st)
        st["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(st["graph"]):
            _own_step(st)


def _order(c):
    return list(range(0, c["layers"], 2)) + list(range(1, c["layers"], 2))


def _own_step(st):
    c, B = st["case"], st["B"]
    for l in _order(c):
        B.paged_attn(st["dims"], st["desc"][l], st["lens"], st["most"], st["q"][l], st["out"][l], _scale(c), st["ws"])


def _own_run(st):
    c, B = st["case"], st["B"]
    if c["kind"] == "prompt":
        B.prompt_attn(st["dims"], st["q"], st["k"], st["v"], st["q_starts"], st["k_lens"], st["out"], _scale(c), st["ws"],
                      k_starts=st["k_starts"])
    elif c["kind"] == "pages":
        k, v = st["kv"].split((c["kv"], c["kv"]), 1)
        B.page_write(st["dims"], st["desc"], k, v, st["seqs"], st["rows"])
        B.page_read(st["dims"], st["desc"], st["k_out"].transpose(0, 1), st["v_out"].transpose(0, 1), st["seqs"], st["rows"])
    elif c["graph"]:
        st["graph"].replay()
    else:
        _own_step(st)


def run(state):
    c = state["case"]
    if own:
        _own_run(state)
    else:
        {"prompt": _plain_prompt, "pages": _plain_pages, "paged": _plain_step}[c["kind"]](state)
    if c["kind"] == "pages":
        return {"k": state["k_out"], "v": state["v_out"]}
    return state["out"]


# ---------------------------------------------------------------- plain forms
def _attend(q, k, v, scale, seen):
    """q [kv][G][n][d], k and v [kv][m][d], all fp32; ``seen [n][m]`` (None: every key): [kv][G][n][d]."""
    kv, G, n, d = q.shape
    s = (q.reshape(kv, G * n, d) @ k.transpose(-1, -2)).view(kv, G, n, -1) * scale
    if seen is not None:
        s = torch.where(seen, s, -math.inf)
    s = (s - s.amax(-1, keepdim=True)).exp()
    return (s.view(kv, G * n, -1) @ v).view(kv, G, n, d) / s.sum(-1, keepdim=True)


def _plain_prompt(st):
    c = st["case"]
    kv, G, d = c["kv"], c["group"], c["d"]
    for s, n in enumerate(st["lens"]):
        q0, T = st["starts"][s], c["past"] + n
        k, v = (x[0, :, q0:q0 + T] if c["packed"] else x[s, :, :T] for x in (st["k"], st["v"]))
        k, v = k.float(), v.float()
        step = max(1, (1 << 28) // (kv * G * T))                         # rows at a time: the logits take a gigabyte
        for a in range(0, n, step):
            b = min(n, a + step)
            q = st["q"][q0 + a:q0 + b].float().view(b - a, kv, G, d).permute(1, 2, 0, 3)
            last = torch.arange(c["past"] + a, c["past"] + b, device="cuda").unsqueeze(1)
            seen = torch.arange(c["past"] + b, device="cuda") <= last
            o = _attend(q, k[:, :c["past"] + b], v[:, :c["past"] + b], _scale(c), seen)
            st["out"][q0 + a:q0 + b] = o.permute(2, 0, 1, 3).reshape(b - a, kv * G, d).to(st["out"].dtype)


def _held(pools, t, page, slot=None):
    """Rows of pages in fp32: [pages][kv][page][d], or [n][kv][d] at the slots ``slot``."""
    at = (page,) if slot is None else (page, slice(None), slot)
    if pools[t + "_exp"] is None:
        return pools[t][at].float()
    code, e = pools[t].view(torch.uint8)[at].contiguous().view(torch.float8_e4m3fn), pools[t + "_exp"][at]
    return code.float() * _power(e).unsqueeze(-1)


def _plain_pages(st):
    c, pools, kv = st["case"], st["pools"], st["case"]["kv"]
    page = st["table"][st["seqs"].long(), st["rows"].long() // c["page"]].long()
    slot = st["rows"].long() % c["page"]
    for t, x in zip("kv", st["kv"].split((kv, kv), 1)):
        if c["dtype"] == "bf16_e4m3":
            code, e = _quantised(x)
            pools[t].view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
            pools[t + "_exp"][page, :, slot] = e
        else:
            pools[t][page, :, slot] = x
    for t in "kv":
        st[t + "_out"].copy_(_held(pools, t, page, slot).transpose(0, 1))


def _plain_step(st):
    c = st["case"]
    kv, G, d = c["kv"], c["group"], c["d"]
    for l in _order(c):
        for s, T in enumerate(st["lens_host"]):
            page = st["table"][s, :-(-T // c["page"])].long()
            k, v = (_held(st["layers"][l], t, page).transpose(0, 1).reshape(kv, -1, d)[:, :T] for t in "kv")
            q = st["q"][l, s].float().view(kv, G, 1, d)
            st["out"][l, s] = _attend(q, k, v, _scale(c), None).view(kv * G, d).to(st["out"].dtype)


# ---------------------------------------------------------------- the work of a pass
def work(case):
    c = case
    d, e, kv, G = c["d"], _bytes(_type(c)), c["kv"], c["group"]
    held = d + 1 if c["dtype"] == "bf16_e4m3" else d * e                # bytes of a row in its page
    if c["kind"] == "pages":
        return {"bytes": 2 * c["tokens"] * kv * (2 * d * e + 2 * held), "flops": 4 * c["tokens"] * kv * d}
    lens = _lengths(c)
    tokens = sum(lens)
    if c["kind"] == "prompt":
        pairs = sum(T * c["past"] + T * (T + 1) // 2 for T in lens)
        return {"bytes": 2 * tokens * kv * G * d * e + 2 * (tokens + c["batch"] * c["past"]) * kv * d * e,
                "flops": 4 * kv * G * d * pairs}
    rows = 2 * c["batch"] * kv * G * d * e
    return {"bytes": c["layers"] * (2 * tokens * kv * held + rows), "flops": c["layers"] * 4 * kv * G * d * tokens}


# ---------------------------------------------------------------- the same in 64 bits
def _softmax_rows(logits):
    w = torch.exp(logits - logits.max(dim=1, keepdim=True).values)
    return w / w.sum(dim=1, keepdim=True)


def _exact_prompt(st):
    c = st["case"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(st["lens"]):
        q0, T = st["starts"][s], c["past"] + n
        for h in range(c["kv"]):
            k, v = ((x[0, h, q0:q0 + T] if c["packed"] else x[s, h, :T]).double() for x in (st["k"], st["v"]))
            kt = k.T.contiguous()
            for g in range(h * c["group"], (h + 1) * c["group"]):
                for a in range(0, n, 4096):
                    b = min(n, a + 4096)
                    m = c["past"] + b                                    # no row of these sees a key behind it
                    z = st["q"][q0 + a:q0 + b, g].double() @ kt[:, :m] / math.sqrt(c["d"])
                    hidden = torch.ones(b - a, m, dtype=torch.bool, device="cuda").triu(c["past"] + a + 1)
                    out[q0 + a:q0 + b, g] = _softmax_rows(z.masked_fill(hidden, -math.inf)) @ v[:m]
    return out


def _two(e):
    """2^e in 64 bits, exactly, for whole numbers."""
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device="cuda")[e.long() + 200]


def _exact_value(code, e):
    """What E4M3 codes and row exponents (both uint8) stand for: sign, four bits of exponent, three of fraction."""
    code = code.long()
    x, f = (code >> 3) & 15, (code & 7).double()
    size = torch.where(x == 0, f * 2.0 ** -9, (8 + f) * _two(x - 10))
    return torch.where(code >= 128, -size, size) * _two(e.long() - 127).unsqueeze(-1)


def _exact_rounded(x):
    """Rows as FP8 with the least power of two that holds them keeps them: four significant bits, ties to even,
    and nothing finer than 2^-9 of that power."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    powers = torch.arange(-126, 128, device="cuda")
    e = (top > 448 * _two(powers)).sum(-1, keepdim=True) - 126           # the least that holds the row
    y = x / _two(e)
    grid = torch.zeros_like(y)
    for p in range(-6, 9):                                               # 2^p <= |y| < 2^(p + 1): steps of 2^(p - 3)
        step = 2.0 ** (p - 3)
        grid = torch.where((y.abs() >= 2.0 ** p) | (p == -6), torch.round(y / step) * step, grid)
    return grid * _two(e)


def _exact_pages(st):
    c, kv = st["case"], st["case"]["kv"]
    x = st["kv"].transpose(0, 1)
    if c["dtype"] == "bf16_e4m3":
        return {"k": _exact_rounded(x[:kv]), "v": _exact_rounded(x[kv:])}
    return {"k": x[:kv].double(), "v": x[kv:].double()}


def _exact_step(st):
    c = st["case"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    P = c["page"]
    for l in range(c["layers"]):
        pools = st["layers"][l]
        for s, T in enumerate(st["lens_host"]):
            t = torch.arange(T, device="cuda")
            page, slot = st["table"][s].long()[t // P], t % P
            for h in range(c["kv"]):
                row = []
                for w in "kv":
                    x = pools[w].view(torch.uint8)[page, h, slot] if c["dtype"] == "bf16_e4m3" else pools[w][page, h, slot]
                    row.append(_exact_value(x, pools[w + "_exp"][page, h, slot]) if c["dtype"] == "bf16_e4m3" else x.double())
                k, v = row
                q = st["q"][l, s, h * c["group"]:(h + 1) * c["group"]].double()
                out[l, s, h * c["group"]:(h + 1) * c["group"]] = _softmax_rows(q @ k.T.contiguous() / math.sqrt(c["d"])) @ v
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"prompt": _exact_prompt, "pages": _exact_pages, "paged": _exact_step}[case["kind"]](st)
