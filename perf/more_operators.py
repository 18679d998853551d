"""Performance cases of the operators for batches of many requests of one model: attention behind prompts that
requests share, and the low-rank adapters that requests bring.

Each case is one call that a serving program makes of the package: a step's queries over a prompt held once and over
each request's own keys, or the adapters' share of a projection whose shared part the program has computed.  ``run``
computes a case in plain torch operations, or with ``own`` set through the package's operators.

Head layouts, widths and lengths are those of the package's own configurations (LLaDA-8B, Dream-7B, the tiny float32
model) and workloads, or generic.
"""
import math
import random

import torch

own = False

# (query heads, key/value heads, head_dim) of the package's configurations, and generic grouped layouts
HEADS = {"llada": (32, 32, 128), "dream": (28, 4, 128), "tiny": (4, 4, 64), "grouped64": (16, 2, 64), "grouped": (32, 8, 128)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# (width in, widths out) of projections: one, queries with keys and values, gate with up, down into the residual
WIDTHS = {"out": (4096, (4096,)), "qkv": (3584, (3584, 512, 512)), "gate_up": (4096, (12288, 12288)), "down": (12288, (4096,)),
          "tiny": (256, (256, 256, 256)), "odd": (333, (201, 77))}


def _shared_case(name, heads, dtype, docs, q, own_keys, prompt, prompts, mix, block, cap, bias, bare, pad):
    c = {"op": "shared", "heads": heads, "dtype": dtype, "docs": docs, "q": q, "own_keys": own_keys, "prompt": prompt,
         "prompts": prompts, "mix": mix, "block": block, "cap": cap, "bias": bias, "bare": bare, "pad": pad}
    return dict(c, name=name) if name else c


def _adapters_case(name, widths, dtype, out, rows, adapters, rank, spread, order, mix):
    c = {"op": "adapters", "widths": widths, "dtype": dtype, "out": out, "rows": rows, "adapters": adapters, "rank": rank,
         "spread": spread, "order": order, "mix": mix}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the tiny float32 model, three requests behind one short prompt, distance biases: latency
        _shared_case("shared_tiny", "tiny", "f32", 3, 1, 37, 150, 1, 1, 1, 0.0, True, 0, 2),
        # one token of 32 requests that continue one long prompt on their own
        _shared_case("shared_token", "dream", "bf16", 32, 1, 512, 8448, 1, 2, 1, 0.0, False, 0, 0),
        # one to four tokens of 24 requests behind three prompts, one request behind none, capped scores
        _shared_case("shared_prompts", "grouped64", "bf16", 24, 4, 300, 2500, 3, 3, 1, 30.0, False, 1, 5),
        # the block rows of a cached denoising step of 16 outputs of one few-shot prompt
        _shared_case("shared_block", "llada", "bf16", 16, 32, 256, 1024, 1, 0, 0, 0.0, False, 0, 0),
        # the same rows behind a long prompt: the prompt's products are most of the work
        _shared_case("shared_block_long", "llada", "bf16", 16, 32, 256, 8448, 1, 0, 0, 0.0, False, 0, 0),
        # questions of unlike lengths read in behind the examples that all of them share, blocks of 32
        _shared_case("shared_questions", "dream", "bf16", 8, 700, 700, 2048, 1, 4, 32, 0.0, False, 0, 37),
        # one row of one request: latency
        _adapters_case("adapters_row", "out", "bf16", "bf16", 1, 4, 16, False, "runs", 1),
        # queries, keys and values of one token of 32 requests, each with an adapter of its own out of 64
        _adapters_case("adapters_token", "qkv", "bf16", "bf16", 32, 64, 16, False, "each", 2),
        # the block rows of eight requests, ranks up to 64, into the float32 residual
        _adapters_case("adapters_block", "down", "bf16", "f32", 256, 8, 64, True, "runs", 3),
        # a long batch through gate and up: bandwidth
        _adapters_case("adapters_long", "gate_up", "bf16", "bf16", 8448, 5, 16, False, "runs", 4),
        # large ranks on prompts of unlike lengths
        _adapters_case("adapters_rank", "out", "bf16", "bf16", 4223, 6, 128, True, "runs", 5),
        # float32 at odd widths, rows of any order, some without an adapter
        _adapters_case("adapters_odd", "odd", "f32", "f32", 777, 7, 8, True, "any", 6),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    mix = rng.randrange(1, 1 << 20)
    if rng.random() < 0.5:
        heads, dtype = rng.choice(list(HEADS)), rng.choice(["bf16", "bf16", "bf16", "f32"])
        most = 1 if dtype == "bf16" else 4
        cap, bias, pad = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3, rng.choice([0, 0, 3, 61])
        kind = rng.choice(["token", "block", "questions"])
        if kind == "token":
            docs = _log(rng, 1, 64)
            return _shared_case(None, heads, dtype, docs, rng.choice([1, 1, 1, 2, 4]), _log(rng, 5, 600), _log(rng, 30, 8448 // most),
                                min(docs, rng.choice([1, 1, 2, 5])), mix, rng.choice([1, 1, 32]), cap, bias, rng.choice([0, 0, 1]), pad)
        if kind == "block":
            docs = _log(rng, 1, 16)
            return _shared_case(None, heads, dtype, docs, rng.choice([16, 32, 33, 64]), _log(rng, 64, 400), _log(rng, 30, 4000 // most),
                                min(docs, rng.choice([1, 1, 2])), mix, rng.choice([0, 0, 32]), cap, bias, rng.choice([0, 0, 1]), pad)
        docs = _log(rng, 1, 12)
        q = _log(rng, 20, min(1300, 1800 // docs) // most)
        return _shared_case(None, heads, dtype, docs, q, q, _log(rng, 30, 2048 // most), min(docs, rng.choice([1, 1, 2])), mix,
                            rng.choice([0, 1, 32]), cap, bias, rng.choice([0, 0, 1]), pad)
    widths, dtype = rng.choice(list(WIDTHS)), rng.choice(["bf16", "bf16", "bf16", "f32"])
    rows = _log(rng, 1, 4200 if dtype == "bf16" else 2000)
    return _adapters_case(None, widths, dtype, rng.choice(["bf16", "f32"]) if dtype == "bf16" else "f32", rows, _log(rng, 1, 24),
                          rng.choice([8, 16, 16, 32, 64]), rng.random() < 0.5, rng.choice(["runs", "runs", "any"]) if rows > 64 else "any", mix)


# ---------------------------------------------------------------- sizes that a case stands for
def _lengths(c):
    """Queries and own keys of each request, the prompt that it continues (-1: none), and the prompts' lengths."""
    rng = random.Random(c["mix"])
    spread = lambda n: n if not c["mix"] else max(1, int(n * rng.uniform(0.3, 1.0)))  # noqa: E731
    keys = [spread(c["own_keys"]) for _ in range(c["docs"])]
    q = [n if c["q"] == c["own_keys"] else min(n, c["q"] if c["block"] != 1 or not c["mix"] else rng.randint(1, c["q"])) for n in keys]
    of = [d * c["prompts"] // c["docs"] for d in range(c["docs"])]
    for d in range(c["bare"]):
        of[c["docs"] // 2 + d] = -1
    return q, keys, of, [spread(c["prompt"]) for _ in range(c["prompts"])]


def _rows_of(c):
    """Each row's adapter (-1: none) and each adapter's rank."""
    rng = random.Random(c["mix"])
    n, R = c["adapters"], c["rank"]
    ranks = [max(1, int(R * rng.uniform(0.1, 1.0))) if c["spread"] else R for _ in range(n)]
    if c["order"] == "each":
        return rng.sample(range(n), c["rows"]), ranks
    if c["order"] == "any":
        return [rng.randint(-1, n - 1) for _ in range(c["rows"])], ranks
    ends = sorted(rng.randint(0, c["rows"]) for _ in range(n - 1))
    return [sum(e <= m for e in ends) for m in range(c["rows"])], ranks


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "shared":
        Hq, Hkv, hd = HEADS[c["heads"]]
        q, keys, of, prompts = _lengths(c)
        pairs = 0
        for a, n, p in zip(q, keys, of):
            seen = [min(n, ((n - a + i) // c["block"] + 1) * c["block"]) if c["block"] else n for i in range(a)]
            pairs += sum(seen) + (a * prompts[p] if p >= 0 else 0)
        held = sum(keys) + sum(prompts[p] for p in set(of) if p >= 0)
        return {"bytes": 2.0 * size * hd * (Hq * sum(q) + Hkv * held), "flops": 4.0 * Hq * hd * pairs}
    K, widths = WIDTHS[c["widths"]]
    which, ranks = _rows_of(c)
    N, S, w = sum(widths), len(widths), 4 if c["out"] == "f32" else 2
    rows = [ranks[a] for a in which if a >= 0]
    used = sum(ranks[a] for a in set(which) if a >= 0)
    return {"bytes": float(len(rows) * K * size + 2 * len(which) * N * w + used * (K * S + N) * size + 4 * len(which)),
            "flops": 2.0 * sum(rows) * (K * S + N)}


# ---------------------------------------------------------------- inputs
def _generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed((seed * 7919 + salt) % (1 << 31))


def _normal(shape, seed, salt, std, dtype):
    return (torch.randn(shape, generator=_generator(seed, salt), device="cuda") * std).to(dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths))]


def _shared_inputs(c, seed):
    Hq, Hkv, hd = HEADS[c["heads"]]
    q, keys, of, prompts = _lengths(c)
    dt, pad = TYPES[c["dtype"]], c["pad"]
    s = {"q": _normal((sum(q) + pad, Hq, hd), seed, 1, 1.3, dt), "out": _normal((sum(q) + pad, Hq, hd), seed, 6, 1.0, dt),
         "k": _normal((sum(keys) + pad, Hkv, hd), seed, 2, 1.3, dt), "v": _normal((sum(keys) + pad, Hkv, hd), seed, 3, 1.3, dt),
         "pk": _normal((sum(prompts) + pad, Hkv, hd), seed, 4, 1.3, dt), "pv": _normal((sum(prompts) + pad, Hkv, hd), seed, 5, 1.3, dt)}
    s["q_start"], s["q_len"], s["kv_start"], s["kv_len"] = _ints(_starts(q)), _ints(q), _ints(_starts(keys)), _ints(keys)
    s["p_start"], s["p_len"], s["of"] = _ints(_starts(prompts)), _ints(prompts), _ints(of)
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device="cuda") if c["bias"] else None
    return s


def _adapters_inputs(c, seed):
    K, widths = WIDTHS[c["widths"]]
    which, ranks = _rows_of(c)
    n, S, N, R = c["adapters"], len(widths), sum(widths), c["rank"]
    dt, ot = TYPES[c["dtype"]], TYPES[c["out"]]
    wide = lambda k: -(-k // 8) * 8  # noqa: E731  rows begin at multiples of 16 bytes
    s = {"x": _normal((c["rows"], wide(K)), seed, 1, 1.0, dt)[:, :K], "base": _normal((c["rows"], wide(N)), seed, 2, 1.0, ot)[:, :N],
         "A": _normal((n, S, R, wide(K)), seed, 3, 1 / math.sqrt(K), dt)[..., :K], "B": _normal((n, N, R), seed, 4, 0.3 / math.sqrt(R), dt),
         "out": _normal((c["rows"], wide(N)), seed, 5, 1.0, ot)[:, :N], "which": _ints(which), "ranks": _ints(ranks) if c["spread"] else None}
    s["scales"] = torch.rand((n,), generator=_generator(seed, 6), device="cuda") * 1.5 + 0.5
    return s


def prepare(case, seed):
    c = case
    if c["op"] == "shared":
        q, keys, _, prompts = _lengths(c)
        return dict(_shared_inputs(c, seed), c=c, max_q=max(q), max_kv=max(keys), max_p=max(prompts))
    return dict(_adapters_inputs(c, seed), c=c, slices=WIDTHS[c["widths"]][1])


# ---------------------------------------------------------------- plain forms
def _plain_shared(s):
    c = s["c"]
    Hq, Hkv, hd = HEADS[c["heads"]]
    n, m, p, g = s["q"].shape[0], s["k"].shape[0], s["pk"].shape[0], Hq // Hkv
    row = torch.arange(n, device="cuda")
    d = torch.searchsorted(s["q_start"], row.int(), right=True) - 1
    at = row - s["q_start"][d]
    covered = at < s["q_len"][d]
    pos = s["kv_len"][d] - s["q_len"][d] + at
    key = torch.arange(m, device="cuda")[None, :] - s["kv_start"][d][:, None]
    sees = (key >= 0) & (key < s["kv_len"][d][:, None]) & covered[:, None]
    if c["block"]:
        sees &= key < (torch.div(pos, c["block"], rounding_mode="floor") + 1)[:, None] * c["block"]
    of = s["of"][d]
    length = torch.where(of >= 0, s["p_len"][of.clamp(min=0)], torch.zeros_like(of))
    pkey = torch.arange(p, device="cuda")[None, :] - s["p_start"][of.clamp(min=0)][:, None]
    psees = (pkey >= 0) & (pkey < length[:, None]) & covered[:, None]
    sees, far = torch.cat([psees, sees], 1), torch.cat([pkey - length[:, None], key], 1) - pos[:, None]
    q = s["q"].float().view(n, Hkv, g, hd).permute(1, 2, 0, 3).reshape(Hkv, g * n, hd)
    k = torch.cat([s["pk"], s["k"]]).float().permute(1, 2, 0).contiguous()
    v = torch.cat([s["pv"], s["v"]]).float().transpose(0, 1).contiguous()
    x = (q @ k).view(Hkv, g, n, p + m)
    x *= 1.0 / math.sqrt(hd)
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    if s["slopes"] is not None:
        x -= s["slopes"].view(Hkv, g, 1, 1) * far.abs().float()
    x.masked_fill_(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    y = (x.view(Hkv, g * n, p + m) @ v).view(Hkv, g, n, hd) / torch.where(total == 0, torch.ones_like(total), total)
    y = y.permute(2, 0, 1, 3).reshape(n, Hq, hd).to(s["out"].dtype)
    s["out"].copy_(torch.where(covered[:, None, None], y, s["out"]))
    return s["out"]


def _plain_adapters(s):
    x, A, B = s["x"].float(), s["A"].float(), s["B"].float()
    n, S, R, K = A.shape
    of = (s["which"][:, None] == torch.arange(n, device="cuda")).float() * s["scales"]
    held = torch.ones((n, R), device="cuda")
    if s["ranks"] is not None:
        held = (torch.arange(R, device="cuda") < s["ranks"][:, None]).float()
    h = (x @ A.reshape(n * S * R, K).T).view(-1, n, S, R) * (of[:, :, None, None] * held[:, None])
    y = [h[:, :, i].reshape(-1, n * R) @ b.permute(0, 2, 1).reshape(n * R, -1) for i, b in enumerate(B.split(s["slices"], 1))]
    s["out"].copy_((s["base"].float() + torch.cat(y, 1)).to(s["out"].dtype))
    return s["out"]


# ---------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["c"]
    if not own:
        return _plain_shared(s) if c["op"] == "shared" else _plain_adapters(s)
    from paper_2608_22646_amd import binding
    if c["op"] == "shared":
        docs = binding.Docs(s["q_start"], s["q_len"], s["kv_start"], s["kv_len"], s["max_q"], s["max_kv"])
        prompts = binding.Prompts(s["p_start"], s["p_len"], s["max_p"], of=s["of"])
        return binding.shared_attention(s["q"], s["k"], s["v"], s["pk"], s["pv"], docs, prompts, block=c["block"], cap=c["cap"],
                                        slopes=s["slopes"], out=s["out"])
    return binding.adapters(s["x"], s["base"], s["A"], s["B"], s["which"], ranks=s["ranks"], scales=s["scales"], slices=s["slices"],
                            out=s["out"])


# ---------------------------------------------------------------- the same in 64 bits
def _exact_shared(c, seed):
    Hq, Hkv, hd = HEADS[c["heads"]]
    s = _shared_inputs(c, seed)
    q, keys, of, prompts = _lengths(c)
    p0, out, q0, k0 = _starts(prompts), s["out"].double(), 0, 0
    for a, b, p in zip(q, keys, of):
        P = prompts[p] if p >= 0 else 0
        behind = slice(p0[p], p0[p] + P) if p >= 0 else slice(0, 0)
        i = P + b - a + torch.arange(a, device="cuda")[:, None]  # positions count from the prompt's first key
        j = torch.arange(P + b, device="cuda")[None, :]
        hidden = (j >= P) & ((j - P) // c["block"] > (i - P) // c["block"]) if c["block"] else None
        for h in range(Hq):
            x = s["q"][q0:q0 + a, h].double() @ torch.cat([s["pk"][behind, h * Hkv // Hq], s["k"][k0:k0 + b, h * Hkv // Hq]]).double().T.contiguous()
            x = x / math.sqrt(hd)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if c["bias"]:
                x = x - 2.0 ** (-8.0 * (h + 1) / Hq) * (i - j).abs()
            if hidden is not None:
                x[hidden] = -math.inf
            out[q0:q0 + a, h] = torch.softmax(x, -1) @ torch.cat([s["pv"][behind, h * Hkv // Hq], s["v"][k0:k0 + b, h * Hkv // Hq]]).double()
        q0, k0 = q0 + a, k0 + b
    return out


def _exact_adapters(c, seed):
    s = _adapters_inputs(c, seed)
    widths = WIDTHS[c["widths"]][1]
    which, ranks = _rows_of(c)
    out = s["base"].double().contiguous()
    for a in sorted(set(which) - {-1}):
        mine, r, first = (s["which"] == a).nonzero()[:, 0], ranks[a], 0
        for i, w in enumerate(widths):
            low = s["x"][mine].double() @ s["A"][a, i, :r].double().T.contiguous()
            out[mine, first:first + w] += float(s["scales"][a]) * (low @ s["B"][a, first:first + w, :r].double().T.contiguous())
            first += w
    return out


def exact(case, seed):
    return _exact_shared(case, seed) if case["op"] == "shared" else _exact_adapters(case, seed)
