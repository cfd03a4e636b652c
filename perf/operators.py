"""Performance cases of the serving step around the compressed cache: the
rotated rows that enter the exact tail, the key bounds and the block selection
of sparse decode, and decode over shared prefixes and selected blocks.

Kinds of cases, each a pass through one operator (or the pair of operators that
is always used together):

* ``rope``   - norm of the query and key heads, rotation by position, and the
               rows' way into the cache (``rope_append``).
* ``bounds`` - per channel the least and the largest key of every block of 64
               tokens, all layers of a prompt (``key_bounds``).
* ``sparse`` - one decode step that attends over the blocks that a bound on the
               logits selects, and over the exact tail (``block_select``, then
               ``decode_parts``).
* ``shared`` - one decode step of a batch whose sequences share a compressed
               prefix and have an exact tail each (``decode_parts``).

Steps run their layers in the order even, then odd, so that the planes a pair
of layers shares are not still in the last-level cache.
"""
import math
import random

import torch

own = False

BLOCK = 64                        # tokens of a selected block
SHARED, RESIDUAL, EXACT = 0, 1, 2
MODES = (4, 3, 1)                 # shared, residual and exact heads of every eight
NEEDLES, NEEDLE_AMP, NEEDLE_CHANNELS = 16, 5.0, 16
MOST = {"rope": 8200 * 48 * 128, "bounds": 16 * 8 * 32768, "sparse": 8 * 8 * 131072, "shared": 8 * 8 * 65536}

# The 8B shape: 32 query heads on 8 KV heads of 128 channels.  Steps take fewer
# layers than the model has, a pipeline stage's share.
M8B = dict(kv=8, group=4, d=128, dtype="bf16")
ROPE = dict(M8B, kind="rope", tokens=1, batch=1, cap=512, norm=False, axes=1, rot=128, interleaved=False, far=32768)
STEP = dict(M8B, layers=8, size=2, topk=16, res_ppm=-1, batch=1, cap=512, graph=False)


def listed():
    return [
        # one token of one sequence: the smallest call, bound by its launch
        dict(ROPE, name="rope_step_8b"),
        # a step of a busy server: normed heads, every sequence at its own position
        dict(ROPE, name="rope_step_b48_norm", tokens=48, batch=48, norm=True),
        # a prompt with images: three axes of positions, normed heads, odd length
        dict(ROPE, name="rope_prompt_8k_3axes", tokens=8191, cap=8192, norm=True, axes=3),
        # the bounds of a 32k prompt, a pipeline stage of 16 layers
        dict(M8B, kind="bounds", name="bounds_8b_32k", layers=16, tokens=32768),
        # the bounds of a short odd prompt of a small fp32 model
        dict(M8B, kind="bounds", name="bounds_f32_1001", kv=4, d=64, dtype="f32", layers=4, tokens=1001),
        # long-context step of one sequence, an eighth of its blocks read, captured in a graph as a server does
        dict(STEP, kind="sparse", name="sparse_8b_32k", layers=16, tmin=32768, tmax=32768, sel=64, first=1, last=2, graph=True),
        # a batch of unlike lengths, FP8 coefficients in blocks of four layers
        dict(STEP, kind="sparse", name="sparse_8b_b16_fp8_quads", batch=16, dtype="bf16_e4m3", size=4, tmin=4096, tmax=16384, sel=32, first=1, last=2),
        # the longest context, eight query heads to a KV head, captured in a graph
        dict(STEP, kind="sparse", name="sparse_70b_131k", group=8, tmin=131072, tmax=131072, sel=128, first=1, last=4, graph=True),
        # a few conversations on a short system prompt, small fp32 model
        dict(STEP, kind="shared", name="shared_f32_1001_b4", layers=2, kv=4, group=2, d=64, topk=8, dtype="f32", batch=4, cap=64, tmin=1001, tmax=1001, graph=True),
        # questions on one long document
        dict(STEP, kind="shared", name="shared_8b_32k_b16", batch=16, tmin=32768, tmax=32768),
        # a busy server on one long system prompt, FP8 coefficients, blocks of four, odd length
        dict(STEP, kind="shared", name="shared_8b_12k_b64_fp8", batch=64, cap=256, dtype="bf16_e4m3", size=4, tmin=12345, tmax=12345),
        # the longest document, eight query heads to a KV head, token-level sets
        dict(STEP, kind="shared", name="shared_70b_131k_b16_tok", layers=4, group=8, batch=16, topk=0, res_ppm=50000, tmin=131072, tmax=131072),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "bounds", "sparse", "sparse", "shared", "shared"])
    d = rng.choice([64, 128, 128])
    kv, group = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    slow = 4 if dtype == "f32" else 1
    if kind == "rope":
        c = dict(ROPE, kv=kv, group=group, d=d, dtype=dtype, norm=rng.random() < 0.6, axes=rng.choice([1, 1, 2, 3]),
                 rot=rng.choice([d, d, d, d // 2, d // 4]), interleaved=rng.random() < 0.3, far=_log_int(rng, 100, 1000000))
        c["tokens"] = _log_int(rng, 1, MOST["rope"] // slow // (kv * (group + 2) * d))
        c["batch"] = rng.choice([1, c["tokens"] if c["tokens"] <= 256 else 1])
        c["cap"] = rng.randint(1, 700) if c["batch"] > 1 else c["tokens"] + rng.randint(0, 300)
        return c
    if kind == "bounds":
        layers = rng.choice([2, 4, 8, 16])
        return dict(M8B, kind=kind, kv=kv, d=d, dtype=dtype, layers=layers, tokens=_log_int(rng, 1, min(131072, MOST["bounds"] // slow // (layers * kv))))
    c = dict(STEP, kind=kind, kv=kv, group=group, d=d, dtype=rng.choice([dtype, "bf16_e4m3"]), size=rng.choice([2, 2, 4]),
             topk=rng.choice([d // 8, d // 8, 5, 24]), cap=rng.choice([64, 200, 512]), graph=rng.random() < 0.5)
    c["layers"] = c["size"] * rng.choice([1, 2]) if c["size"] == 4 else rng.choice([2, 4, 8])
    if rng.random() < 0.25:
        c["topk"], c["res_ppm"] = 0, rng.choice([10000, 50000, 100000])
    room = MOST[kind] // slow // (c["layers"] * kv)
    if kind == "sparse":
        c["batch"] = rng.choice([1, 1, 2, 5, 16])
        c["tmax"] = _log_int(rng, 100, max(200, min(131072, room // c["batch"])))
        c["tmin"] = max(1, c["tmax"] // 4) if c["batch"] > 1 else c["tmax"]
        c["first"], c["last"] = rng.choice([0, 1, 2]), rng.choice([1, 2, 4])
        c["sel"] = max(c["first"] + c["last"], _log_int(rng, 4, 128))
    else:
        c["batch"] = rng.choice([2, 3, 8, 16, 33, 64])
        c["tmin"] = c["tmax"] = _log_int(rng, 100, max(200, min(131072, room // max(1, c["batch"] * group // 32))))
    return c


# ---------------------------------------------------------------- inputs
def _gen(seed, *tags):
    return torch.Generator("cuda").manual_seed(random.Random("%d %s" % (seed, tags)).getrandbits(62))


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _coef_type(c):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "bf16_e4m3": torch.float8_e4m3fn}[c["dtype"]]


def _bytes(t):
    return torch.empty(0, dtype=t).element_size()


def _rand(c, seed, tag, *shape):
    return torch.randn(*shape, generator=_gen(seed, tag), device="cuda").to(_type(c))


def _depth(c, g, size, T):
    """K and V of a block's layers, [2][size][kv][T][d]: along depth a first-order
    autoregression, one correlation a head, with needle tokens whose channels spike in one layer."""
    d, kv = c["d"], c["kv"]
    rho = 0.75 + 0.20 * torch.rand(kv, 1, 1, generator=g, device="cuda")
    x = torch.empty(2, size, kv, T, d, dtype=_type(c), device="cuda")
    y = torch.randn(2, kv, T, d, generator=g, device="cuda")
    x[:, 0] = y
    for n in range(1, size):
        y = rho * y + (1 - rho * rho).sqrt() * torch.randn(2, kv, T, d, generator=g, device="cuda")
        x[:, n] = y
    m = min(NEEDLES, T)
    pos = torch.randperm(T, generator=g, device="cuda")[:m].view(1, m, 1)
    chan = torch.rand(kv, m, d, generator=g, device="cuda").argsort(-1)[..., :NEEDLE_CHANNELS]
    layer = torch.randint(size, (kv, m, 1), generator=g, device="cuda")
    x[:, layer, torch.arange(kv, device="cuda").view(kv, 1, 1), pos, chan] += NEEDLE_AMP
    return x


def _pad(n, to=256):
    return -(-n // to) * to


def _planes(c, mode, T):
    """Byte offset and length of every plane of a unit's segment, and the segment's bytes."""
    d, e, f, size = c["d"], _bytes(_type(c)), _bytes(_coef_type(c)), c["size"]
    coef = _pad(T * d, 1024) if f == 1 else T * d * f
    if mode == EXACT:
        parts = [("k%d" % i, T * d * e) for i in range(size)] + [("v%d" % i, T * d * e) for i in range(size)]
    else:
        parts = [("mk", coef), ("mv", coef)]
        if mode == RESIDUAL and c["res_ppm"] >= 0:
            n = -(-T * c["res_ppm"] // 1000000)
            rows = n * (size - 1) * d * f
            parts += [("mask", -(-T // 32) * 4), ("count", (-(-T // 128) + 1) * 4), ("hk", rows), ("hv", rows)]
        elif mode == RESIDUAL:
            i = T * c["topk"] * (1 if size == 2 else 2)
            v = T * c["topk"] * f
            parts += [("ik", i), ("xk", v), ("iv", i), ("xv", v)]
    at, off = {}, 0
    for name, n in parts:
        at[name] = (off, n)
        off += _pad(n)
    return at, off


def _dct4():
    n = torch.arange(4, dtype=torch.float64, device="cuda")
    return torch.stack([torch.cos(math.pi * (2 * n + 1) * j / 8) / math.sqrt(2) for j in range(4)])


def _stored(c, x):
    x = x.clamp(-448, 448) if c["dtype"] == "bf16_e4m3" else x
    return x.to(_coef_type(c))


def _write_group(c, g, mode, heads, x, at, seg):
    """Fills the segments ``seg [n][bytes]`` of neighbouring heads of one mode."""
    n, T, d = len(heads), x.shape[3], c["d"]

    def put(name, t):
        o, m = at[name]
        if m:
            seg[:, o:o + m] = t.contiguous().view(n, -1).view(torch.uint8)

    kept = None
    for i, t in enumerate("kv"):
        y = x[i][:, heads]                               # [size][n][T][d]
        if mode == EXACT:
            for p in range(c["size"]):
                put("%s%d" % (t, p), y[p])
            continue
        mean = _stored(c, y.float().mean(0))
        if c["dtype"] == "bf16_e4m3":                    # 1 KB blocks of 1024 / d rows, rows r and r + half side by side
            half = 512 // d
            m = torch.zeros(n, _pad(T, 2 * half), d, dtype=torch.uint8, device="cuda")
            m[:, :T] = mean.view(torch.uint8)
            mean = m.view(n, -1, 2, half, d // 8, 8).permute(0, 1, 3, 4, 2, 5)
        put("m" + t, mean)
        if mode == SHARED:
            continue
        if c["size"] == 2:
            z = ((y[0].float() - y[1].float()) / 2).unsqueeze(-1)
        else:
            f = _dct4().float()
            z = torch.stack([sum(f[j][p] * y[p].float() for p in range(4)) for j in (1, 2, 3)], -1)
        if c["res_ppm"] >= 0:
            ns = -(-T * c["res_ppm"] // 1000000)
            if kept is None:                             # the tokens that differ most along depth
                kept = z.square().sum((-1, -2)).topk(ns, dim=1)[1].sort(1)[0]
                mask = torch.zeros(n, _pad(T, 128), dtype=torch.int64, device="cuda").scatter_(1, kept, 1)
                bits = (mask[:, :_pad(T, 32)].view(n, -1, 32) << torch.arange(32, device="cuda")).sum(-1)
                put("mask", torch.where(bits >= 1 << 31, bits - (1 << 32), bits).to(torch.int32))
                count = mask.view(n, -1, 128).sum(-1).cumsum(1)
                put("count", torch.cat([torch.zeros_like(count[:, :1]), count], 1).to(torch.int32))
            rows = z.gather(1, kept.view(n, ns, 1, 1).expand(n, ns, d, z.shape[-1]))
            put("h" + t, _stored(c, rows.transpose(-1, -2)))
        else:
            code = z.abs().flatten(2).topk(c["topk"], dim=-1)[1].sort(-1)[0]
            put("x" + t, _stored(c, z.flatten(2).gather(-1, code)))
            if c["size"] == 2:
                put("i" + t, code.to(torch.uint8))
            else:
                put("i" + t, (4 * (code // 3) + code % 3 + 1).to(torch.int16))


def _cache(c, seed, lens):
    """A compressed cache as its prefill leaves it: the buffer, modes and segment offsets
    [batch][blocks][kv], and per (sequence, block) the groups (mode, first head, heads) of equal mode."""
    kv, nb = c["kv"], c["layers"] // c["size"]
    count = [max(0, round(kv * m / sum(MODES))) for m in MODES]
    count[SHARED] = kv - count[RESIDUAL] - count[EXACT]
    r = random.Random("modes %d" % seed)
    groups, off, total = {}, torch.zeros(len(lens), nb, kv, dtype=torch.int64), 0
    modes = torch.zeros(len(lens), nb, kv, dtype=torch.uint8)
    for s, T in enumerate(lens):
        for b in range(nb):
            order = [m for m in range(3) if count[m]]
            r.shuffle(order)
            h = 0
            groups[s, b] = []
            for m in order:
                groups[s, b].append((m, h, count[m]))
                for i in range(h, h + count[m]):
                    modes[s, b, i], off[s, b, i] = m, total
                    total += _planes(c, m, T)[1]
                h += count[m]
    buf = torch.zeros(max(total, 256), dtype=torch.uint8, device="cuda")
    bounds = []
    for s, T in enumerate(lens):
        for b in range(nb):
            g = _gen(seed, "cache", s, b)
            x = _depth(c, g, c["size"], T)
            if c["kind"] == "sparse":
                bounds.append(_bounds(x[0].float(), T).to(_type(c)))
            for m, h, n in groups[s, b]:
                at, size = _planes(c, m, T)
                o = int(off[s, b, h])
                _write_group(c, g, m, list(range(h, h + n)), x, at, buf[o:o + n * size].view(n, size))
    return dict(buf=buf, modes=modes, off=off, groups=groups, lens=lens, per=bounds)


def _lens(c, seed):
    r = random.Random("lens %d" % seed)
    return [r.randint(c["tmin"], c["tmax"]) for _ in range(c["batch"] if c["kind"] == "sparse" else 1)]


def _scale(c):
    return 1.0 / math.sqrt(c["d"])


def prepare(case, seed):
    c = case
    st = dict(case=c)
    if c["kind"] == "rope":
        n, kv, hq, d = c["tokens"], c["kv"], c["kv"] * c["group"], c["d"]
        st["qkv"] = _rand(c, seed, "qkv", n, (hq + 2 * kv) * d)          # one projection's output, rows of all heads
        r = random.Random("positions %d" % seed)
        st["pos"] = torch.stack([torch.randint(r.randint(1, c["far"]), (n,), generator=_gen(seed, "pos", a), device="cuda")
                                 for a in range(c["axes"])]).to(torch.int32)
        st["freq"] = 500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
        pairs = c["rot"] // 2
        st["axis"] = [i * c["axes"] // pairs for i in range(pairs)]       # low frequencies on the last axis
        if c["norm"]:
            st["wq"], st["wk"] = ((1 + 0.2 * _rand(c, seed, t, d).float()).to(_type(c)) for t in ("q norm", "k norm"))
        many = c["batch"] > 1
        st["seqs"] = torch.arange(n, dtype=torch.int32, device="cuda") if many else torch.zeros(n, dtype=torch.int32, device="cuda")
        st["rows"] = torch.randint(c["cap"], (n,), generator=_gen(seed, "rows"), device="cuda").to(torch.int32) if many else \
            torch.arange(n, dtype=torch.int32, device="cuda") + (c["cap"] - n) // 2
        st["k"], st["v"] = (torch.zeros(c["batch"], kv, c["cap"], d, dtype=_type(c), device="cuda") for _ in range(2))
        st["q"] = torch.empty(n, hq, d, dtype=_type(c), device="cuda")
        st["axes"] = torch.tensor(st["axis"], device="cuda")
    elif c["kind"] == "bounds":
        st["k"] = [_rand(c, seed, ("k", l), c["kv"], c["tokens"], c["d"]) for l in range(c["layers"])]
        st["bounds"] = torch.empty(c["layers"], c["kv"], -(-c["tokens"] // BLOCK), 2, c["d"], dtype=_type(c), device="cuda")
    else:
        lens, L, kv = _lens(c, seed), c["layers"], c["kv"]
        cache = st["cache"] = _cache(c, seed, lens)
        st["q"] = _rand(c, seed, "q", L, c["batch"], kv * c["group"], c["d"]) * 2.0
        st["out"] = torch.empty_like(st["q"])
        st["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        r = random.Random("tail %d" % seed)
        st["tail_lens"] = torch.tensor([r.randint(1, c["cap"]) for _ in range(c["batch"])], dtype=torch.int32, device="cuda")
        st["tail"] = _rand(c, seed, "tail", L, 2, c["batch"], kv, c["cap"], c["d"])
        st["off"] = cache["off"].to("cuda")
        flat = torch.zeros(_pad(cache["modes"].numel(), 4), dtype=torch.uint8)
        flat[:cache["modes"].numel()] = cache["modes"].flatten()
        st["modes"] = flat.to("cuda")
        if c["kind"] == "sparse":
            nb = -(-max(lens) // BLOCK)
            st["bounds"] = torch.zeros(L, c["batch"], kv, nb, 2, c["d"], dtype=_type(c), device="cuda")
            per, blocks = cache.pop("per"), L // c["size"]
            for s, T in enumerate(lens):
                for b in range(blocks):
                    st["bounds"][b * c["size"]:(b + 1) * c["size"], s, :, :-(-T // BLOCK)] = per[s * blocks + b]
            st["blocks"] = torch.empty(L, c["batch"], kv, c["sel"], dtype=torch.int32, device="cuda")
            st["counts"] = torch.empty(L, c["batch"], kv, dtype=torch.int32, device="cuda")
    if own:
        _handles(st)
    return st


def _handles(st):
    """What a program of this framework keeps between steps: descriptors, workspaces, a captured step."""
    from paper_2607_06519_amd import binding as B
    c = st["case"]
    hq = c["kv"] * c["group"]
    st["B"] = B
    if c["kind"] == "rope":
        st["dims"] = B.dims(2, c["kv"], hq, c["d"], 0, c["dtype"])
        st["rope"] = B.rope(c["rot"], st["freq"], st["pos"], axis=st["axis"], interleaved=c["interleaved"])
        return
    if c["kind"] == "bounds":
        st["dims"] = B.dims(c["layers"], c["kv"], hq, c["d"], 0, c["dtype"])
        return
    tok = c["res_ppm"] >= 0
    dims = st["dims"] = B.dims(c["layers"], c["kv"], hq, c["d"], c["topk"], c["dtype"], 0 if c["size"] == 2 else 2,
                               B.RES_TOKENS if tok else B.RES_CHANNELS, c["res_ppm"] if tok else 0)
    T = max(st["cache"]["lens"])
    kind = B.PART_SHARED if c["kind"] == "shared" else B.PART_BLOCKS
    args = dict(seq_lens=st["lens"], max_seq_len=T, modes=st["modes"], seg_offsets=st["off"], cache=st["cache"]["buf"])
    st["parts"], st["tails"] = [], []
    for l in range(c["layers"]):
        if kind == B.PART_BLOCKS:
            args.update(blocks=st["blocks"][l], counts=st["counts"][l], n_sel=c["sel"])
        st["parts"].append([B.part(kind, **args)])
        k, v = st["tail"][l]
        st["tails"].append(B.Tail(st["tail_lens"].data_ptr(), c["cap"], k.data_ptr(), v.data_ptr()))
    st["ws"] = torch.empty(B.decode_parts_workspace(dims, c["batch"], st["parts"][0], c["cap"]) // 4 + 64, dtype=torch.float32, device="cuda")
    if kind == B.PART_BLOCKS:
        st["select_ws"] = torch.empty(B.block_select_workspace(dims, c["batch"], T) // 4 + 64, dtype=torch.float32, device="cuda")
    if c["graph"]:
        _own_step(st)
        st["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(st["graph"]):
            _own_step(st)


def _order(c):
    return list(range(0, c["layers"], 2)) + list(range(1, c["layers"], 2))


def _own_step(st):
    c, B, dims = st["case"], st["B"], st["dims"]
    for l in _order(c):
        if c["kind"] == "sparse":
            B.block_select(dims, c["batch"], st["lens"], max(st["cache"]["lens"]), st["bounds"][l], st["q"][l], c["first"], c["last"],
                           c["sel"], st["blocks"][l], st["counts"][l], st["select_ws"])
        B.decode_parts(dims, c["batch"], st["parts"][l], st["tails"][l], l, st["q"][l], st["out"][l], _scale(c), st["ws"])


def _own_run(st):
    c, B = st["case"], st["B"]
    if c["kind"] == "rope":
        hq, kv, d = c["kv"] * c["group"], c["kv"], c["d"]
        q, k, v = st["qkv"].view(c["tokens"], hq + 2 * kv, d).split((hq, kv, kv), 1)
        B.rope_append(st["dims"], st["rope"], q, k, v, st["q"], st["seqs"], st["rows"], st["k"], st["v"],
                      q_norm=st.get("wq"), k_norm=st.get("wk"), eps=1e-6)
    elif c["kind"] == "bounds":
        B.key_bounds(st["dims"], c["tokens"], st["k"], list(st["bounds"]), st["bounds"].shape[2])
    elif c["graph"]:
        st["graph"].replay()
    else:
        _own_step(st)


def run(state):
    c = state["case"]
    if own:
        _own_run(state)
    else:
        {"rope": _plain_rope, "bounds": _plain_bounds, "sparse": _plain_step, "shared": _plain_step}[c["kind"]](state)
    if c["kind"] == "rope":
        return {"q": state["q"], "k": state["k"], "v": state["v"]}
    if c["kind"] == "bounds":
        return state["bounds"]
    if c["kind"] == "sparse":
        return {"out": state["out"], "blocks": state["blocks"], "counts": state["counts"]}
    return state["out"]


# ---------------------------------------------------------------- plain forms
def _plain_rope(st):
    c = st["case"]
    n, hq, kv, d, rot = c["tokens"], c["kv"] * c["group"], c["kv"], c["d"], c["rot"]
    q, k, v = st["qkv"].view(n, hq + 2 * kv, d).split((hq, kv, kv), 1)
    angle = st["pos"][st["axes"]].T.double() * st["freq"]                # [n][pairs]; far positions need 64 bits
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        y = x.clone()
        if c["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
        return y.to(_type(c))

    st["q"].copy_(turned(q, st.get("wq")))
    at = (st["seqs"].long(), slice(None), st["rows"].long())
    st["k"][at] = turned(k, st.get("wk"))
    st["v"][at] = v


def _bounds(k, T):
    """[..][T][d] in fp32 -> [..][blocks][2][d]: least and largest value of each channel."""
    nb = -(-T // BLOCK)
    pad = k[..., -1:, :].expand(*k.shape[:-2], nb * BLOCK - T, k.shape[-1])   # repeats of a row change neither
    x = torch.cat([k, pad], -2).unflatten(-2, (nb, BLOCK))
    return torch.stack([x.amin(-2), x.amax(-2)], -2)


def _plain_bounds(st):
    T = st["case"]["tokens"]
    for l, k in enumerate(st["k"]):
        st["bounds"][l] = _bounds(k.float(), T).to(k.dtype)


def _plane(c, cache, s, b, group, name, dtype):
    """A plane of neighbouring heads of one mode as it lies in the buffer, [n][elements]."""
    mode, h, n = group
    at, size = _planes(c, mode, cache["lens"][s])
    o, m = at[name]
    base = int(cache["off"][s, b, h])
    return cache["buf"][base:base + n * size].view(n, size)[:, o:o + m].view(dtype)


def _rows(c, cache, s, b, group, p, tok):
    """K and V rows [n][m][d] in fp32 of layer p of a block, at tokens ``tok [n][m]`` (None: all)."""
    mode, _, n = group
    T, d = cache["lens"][s], c["d"]

    def pick(x):
        return x if tok is None else x[torch.arange(n, device="cuda").unsqueeze(1), tok]

    if c["size"] == 2:
        w = torch.tensor([1.0 - 2.0 * p], device="cuda")
    else:
        w = _dct4()[1:, p].float()
    out = []
    for t in "kv":
        if mode == EXACT:
            out.append(pick(_plane(c, cache, s, b, group, "%s%d" % (t, p), _type(c)).view(n, T, d)).float())
            continue
        m = _plane(c, cache, s, b, group, "m" + t, _coef_type(c))
        if c["dtype"] == "bf16_e4m3":
            half = 512 // d
            m = m.view(torch.uint8).view(n, -1, half, d // 8, 2, 8).permute(0, 1, 4, 2, 3, 5).reshape(n, -1, d)[:, :T].view(torch.float8_e4m3fn)
            x = pick(m.view(torch.uint8)).contiguous().view(torch.float8_e4m3fn).float()
        else:
            x = pick(m.view(n, T, d)).float()
        if mode == RESIDUAL and c["res_ppm"] >= 0:
            bits = _plane(c, cache, s, b, group, "mask", torch.int32)
            in_set = ((bits.unsqueeze(-1) >> torch.arange(32, device="cuda")) & 1).view(n, -1)[:, :T]
            rank = (in_set.cumsum(1) - 1).clamp(min=0)
            h = _plane(c, cache, s, b, group, "h" + t, _coef_type(c)).view(n, -1, c["size"] - 1, d).float()
            h = (h * w.view(-1, 1)).sum(2)
            x = x + pick(in_set.unsqueeze(-1)) * h[torch.arange(n, device="cuda").unsqueeze(1), pick(rank.unsqueeze(-1)).squeeze(-1)]
        elif mode == RESIDUAL:
            code = pick(_plane(c, cache, s, b, group, "i" + t, torch.uint8 if c["size"] == 2 else torch.int16).view(n, T, -1)).long()
            val = pick(_plane(c, cache, s, b, group, "x" + t, _coef_type(c)).view(n, T, -1).view(torch.uint8).view(n, T, -1))
            val = val.contiguous().view(_coef_type(c)).float()
            if c["size"] == 2:
                x = x.scatter_add(-1, code, val * w)
            else:
                x = x.scatter_add(-1, code >> 2, val * w[(code & 3) - 1])
        out.append(x)
    return out


def _attend(q, k, v, tk, tv, lens, scale):
    """q [n][b][G][d]; k, v [n][m][d] for all of b; the sequences' tails tk, tv [b][n][cap][d] with ``lens`` rows."""
    n, b, G, d = q.shape
    s = (q.reshape(n, b * G, d) @ k.transpose(-1, -2)).view(n, b, G, -1) * scale
    tk, tv = tk.float().transpose(0, 1), tv.float().transpose(0, 1)
    held = torch.arange(tk.shape[2], device="cuda") < lens.view(1, b, 1, 1)
    t = torch.where(held, (q @ tk.transpose(-1, -2)) * scale, -math.inf)
    top = torch.maximum(s.amax(-1, keepdim=True), t.amax(-1, keepdim=True))
    s, t = (s - top).exp(), (t - top).exp()
    o = (s.reshape(n, b * G, -1) @ v).view(n, b, G, d) + t @ tv
    return (o / (s.sum(-1, keepdim=True) + t.sum(-1, keepdim=True))).transpose(0, 1)


def _plain_select(st, l):
    """The blocks of largest bound on a logit, counted from each head's best block, the largest over a group."""
    c, bound = st["case"], st["bounds"][l].double()
    bsz, kv, nb, _, d = bound.shape
    q = st["q"][l].view(bsz, kv, -1, d).double()
    score = q.clamp(min=0) @ bound[..., 1, :].transpose(-1, -2) + q.clamp(max=0) @ bound[..., 0, :].transpose(-1, -2)
    held = ((st["lens"] + BLOCK - 1) // BLOCK).view(bsz, 1, 1)
    j = torch.arange(nb, device="cuda")
    score = torch.where((j < held).unsqueeze(-2), score, -math.inf)
    rank = (score - score.amax(-1, keepdim=True)).amax(-2)
    rank = torch.where((j < c["first"]) | (j >= held - c["last"]), math.inf, rank)
    rank = torch.where(j < held, rank, -math.inf)
    best = rank.sort(dim=-1, descending=True, stable=True)[1][..., :c["sel"]]
    count = held.clamp(max=c["sel"]).expand(bsz, kv, 1)
    best = torch.cat([best, best.new_full((bsz, kv, c["sel"] - best.shape[-1]), nb)], -1)
    best = torch.where(torch.arange(c["sel"], device="cuda") < count, best, nb).sort(-1)[0]
    st["blocks"][l] = torch.where(best < nb, best, -1).to(torch.int32)
    st["counts"][l] = count.squeeze(-1).to(torch.int32)


def _plain_step(st):
    c, cache = st["case"], st["cache"]
    G, d = c["group"], c["d"]
    for l in _order(c):
        b, p = l // c["size"], l % c["size"]
        q = st["q"][l].view(c["batch"], c["kv"], G, d)
        out = st["out"][l].view(c["batch"], c["kv"], G, d)
        tk, tv = st["tail"][l]
        if c["kind"] == "shared":
            for group in cache["groups"][0, b]:
                h = slice(group[1], group[1] + group[2])
                k, v = _rows(c, cache, 0, b, group, p, None)
                out[:, h] = _attend(q[:, h].float().transpose(0, 1), k, v, tk[:, h], tv[:, h], st["tail_lens"], _scale(c)).to(out.dtype)
            continue
        _plain_select(st, l)
        for s, T in enumerate(cache["lens"]):
            m = min(c["sel"], -(-T // BLOCK))
            for group in cache["groups"][s, b]:
                h = slice(group[1], group[1] + group[2])
                tok = (st["blocks"][l, s, h, :m].long().unsqueeze(-1) * BLOCK + torch.arange(BLOCK, device="cuda")).flatten(1)
                held = (tok < T).unsqueeze(-1)
                k, v = _rows(c, cache, s, b, group, p, tok.clamp(max=T - 1))
                o = _attend_held(q[s, h].float(), k, v, held, tk[s, h], tv[s, h], st["tail_lens"][s], _scale(c))
                out[s, h] = o.to(out.dtype)


def _attend_held(q, k, v, held, tk, tv, n, scale):
    """q [n][G][d] over rows k, v [n][m][d] where ``held [n][m][1]``, and a tail's first ``n`` rows."""
    rows = torch.arange(tk.shape[1], device="cuda").view(1, -1, 1) < n
    k, v = torch.cat([k, tk.float()], 1), torch.cat([v, tv.float()], 1)
    held = torch.cat([held, rows.expand(k.shape[0], -1, 1)], 1).transpose(-1, -2)
    s = torch.where(held, q @ k.transpose(-1, -2) * scale, -math.inf)
    s = (s - s.amax(-1, keepdim=True)).exp()
    return s @ v / s.sum(-1, keepdim=True)


# ---------------------------------------------------------------- the work of a pass
def _read(c):
    """Bytes per token that one layer reads of its KV heads, in the shares of the modes."""
    d, e, f, k, kv = c["d"], _bytes(_type(c)), _bytes(_coef_type(c)), c["topk"], c["kv"]
    ent = 2 * k * (f + c["size"] // 2)
    if c["res_ppm"] >= 0:
        ent = 2 * (c["size"] - 1) * d * f * c["res_ppm"] / 1e6
    count = [round(kv * m / sum(MODES)) for m in MODES]
    count[SHARED] = kv - count[RESIDUAL] - count[EXACT]
    return count[SHARED] * 2 * d * f + count[RESIDUAL] * (2 * d * f + ent) + count[EXACT] * 2 * d * e


def work(case):
    c = case
    d, e, kv, G = c["d"], _bytes(_type(c)), c["kv"], c["group"]
    if c["kind"] == "rope":
        values = c["tokens"] * kv * (G + 2) * d
        return {"bytes": 2 * values * e, "flops": 6 * values}
    if c["kind"] == "bounds":
        keys = c["layers"] * kv * c["tokens"] * d
        return {"bytes": keys * e + c["layers"] * kv * -(-c["tokens"] // BLOCK) * 2 * d * e, "flops": 2 * keys}
    rows = 2 * c["batch"] * kv * G * d * e
    tail = c["batch"] * kv * (c["cap"] + 1) / 2
    T = (c["tmin"] + c["tmax"]) / 2
    if c["kind"] == "shared":
        tokens, at = T, c["batch"] * T
        look = 0
    else:
        tokens = at = c["batch"] * min(T, c["sel"] * BLOCK)
        look = c["batch"] * kv * math.ceil(T / BLOCK) * 2 * d
    return {"bytes": int(c["layers"] * (tokens * _read(c) + tail * 2 * d * e + rows + look * e)),
            "flops": int(c["layers"] * (4 * G * d * (kv * at + tail) + 2 * G * look))}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_rope(st):
    c = st["case"]
    n, hq, kv, d, rot = c["tokens"], c["kv"] * c["group"], c["kv"], c["d"], c["rot"]
    x = st["qkv"].double().view(n, hq + 2 * kv, d)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       torch.stack([st["pos"][a].double() * f for a, f in zip(st["axis"], st["freq"])], 1))
    heads = []
    for h in range(hq + kv):
        y, w = x[:, h], st.get("wq" if h < hq else "wk")
        if w is not None:
            y = y / (y.square().sum(1, keepdim=True) / d + 1e-6).sqrt() * w.double()
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(y[:, lo].contiguous(), y[:, hi].contiguous()) * turn
        y = y.clone()
        y[:, lo], y[:, hi] = z.real, z.imag
        heads.append(y)
    k, v = (torch.zeros(st["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for h in range(kv):
        k[st["seqs"].long(), h, st["rows"].long()] = heads[hq + h]
        v[st["seqs"].long(), h, st["rows"].long()] = x[:, hq + kv + h]
    return {"q": torch.stack(heads[:hq], 1), "k": k, "v": v}


def _exact_unit(c, cache, s, b, h, p):
    """K and V [T][d] in 64 bits of one head's unit, from its bytes."""
    T, d, size = cache["lens"][s], c["d"], c["size"]
    mode = int(cache["modes"][s, b, h])
    at, total = _planes(c, mode, T)
    seg = cache["buf"][int(cache["off"][s, b, h]):][:total]

    def plane(name, dtype):
        o, m = at[name]
        return seg[o:o + m].clone().view(dtype)

    f = _dct4()
    weight = [1.0 if p == 0 else -1.0] if size == 2 else [float(f[j][p]) for j in (1, 2, 3)]
    res = []
    for t in "kv":
        if mode == EXACT:
            res.append(plane("%s%d" % (t, p), _type(c)).double().view(T, d))
            continue
        m = plane("m" + t, _coef_type(c)).double()
        if c["dtype"] == "bf16_e4m3":                    # where the header says that channel ch of row r sits
            R = 1024 // d
            r, ch = torch.arange(T, device="cuda").view(T, 1), torch.arange(d, device="cuda").view(1, d)
            m = m[1024 * (r // R) + 16 * ((r % (R // 2)) * (d // 8) + ch // 8) + 8 * ((r % R) // (R // 2)) + ch % 8]
        x = m.view(T, d).clone()
        if mode == RESIDUAL and c["res_ppm"] >= 0:
            word = plane("mask", torch.int32).long() & 0xFFFFFFFF
            r = torch.arange(T, device="cuda")
            kept = torch.nonzero((word[r // 32] >> (r % 32)) & 1).flatten()
            z = plane("h" + t, _coef_type(c)).double().view(-1, size - 1, d)
            for j in range(size - 1):
                x[kept] += weight[j] * z[:, j]
        elif mode == RESIDUAL:
            code = plane("i" + t, torch.uint8 if size == 2 else torch.int16).long().view(T, -1)
            val = plane("x" + t, _coef_type(c)).double().view(T, -1)
            for j in range(size - 1):
                dense = torch.zeros(T, d, dtype=torch.float64, device="cuda")
                mine = torch.ones_like(code, dtype=torch.bool) if size == 2 else (code % 4) == j + 1
                dense.scatter_add_(1, code if size == 2 else code // 4, torch.where(mine, val, 0.0))
                x += weight[j] * dense
        res.append(x)
    return res


def _exact_blocks(st, l, s, h):
    c, T = st["case"], st["cache"]["lens"][s]
    nb = -(-T // BLOCK)
    lo, hi = st["bounds"][l, s, h, :nb, 0].double(), st["bounds"][l, s, h, :nb, 1].double()
    key = None
    for g in range(c["group"]):
        q = st["q"][l, s, h * c["group"] + g].double()
        bound = torch.where(q > 0, q * hi, q * lo).sum(1)
        bound = bound - bound.max()
        key = bound if key is None else torch.maximum(key, bound)
    key = key.tolist()
    forced = set(range(min(c["first"], nb))) | set(range(max(0, nb - c["last"]), nb))
    rest = sorted((j for j in range(nb) if j not in forced), key=lambda j: (-key[j], j))
    return sorted((sorted(forced) + rest)[:c["sel"]])


def _exact_step(st):
    c, cache = st["case"], st["cache"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    blocks = torch.full(st["blocks"].shape, -1, dtype=torch.int32) if c["kind"] == "sparse" else None
    counts = torch.zeros(st["counts"].shape, dtype=torch.int32) if c["kind"] == "sparse" else None
    G = c["group"]
    for l in range(c["layers"]):
        tk, tv = st["tail"][l]
        for h in range(c["kv"]):
            unit = None
            for s in range(c["batch"]):
                if unit is None or c["kind"] == "sparse":
                    unit = _exact_unit(c, cache, s, l // c["size"], h, l % c["size"])
                k, v = unit
                if c["kind"] == "sparse":
                    sel = _exact_blocks(st, l, s, h)
                    blocks[l, s, h, :len(sel)] = torch.tensor(sel, dtype=torch.int32)
                    counts[l, s, h] = len(sel)
                    at = torch.cat([torch.arange(j * BLOCK, min(len(k), (j + 1) * BLOCK)) for j in sel]).to("cuda")
                    k, v = k[at], v[at]
                n = int(st["tail_lens"][s])
                k, v = torch.cat([k, tk[s, h, :n].double()]), torch.cat([v, tv[s, h, :n].double()])
                q = st["q"][l, s, h * G:(h + 1) * G].double()
                prob = torch.softmax(q @ k.T.contiguous() / math.sqrt(c["d"]), 1)
                out[l, s, h * G:(h + 1) * G] = prob @ v
    return {"out": out, "blocks": blocks.to("cuda"), "counts": counts.to("cuda")} if c["kind"] == "sparse" else out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(st)
    if case["kind"] == "bounds":
        return torch.stack([torch.stack([torch.stack([x.amin(1), x.amax(1)], 1) for x in k.double().split(BLOCK, 1)], 1) for k in st["k"]])
    return _exact_step(st)
