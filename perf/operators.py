"""Performance cases of the stand-alone operators: rotary positions, attention over packed documents, sampling.

Each case is one call that a serving program makes of the package: rotating a
step's queries and keys, attending over the requests of a ragged batch, drawing
the block's tokens from the head's logits.  ``run`` computes a case in plain
torch operations, or with ``own`` set through the package's operators.

Head layouts, vocabularies and lengths are those of the package's own
configurations (LLaDA-8B, Dream-7B, the tiny float32 model) and workloads.
"""
import math
import random

import torch

own = False

# (query heads, key/value heads, head_dim) of the package's configurations, and generic grouped layouts
HEADS = {"llada": (32, 32, 128), "dream": (28, 4, 128), "tiny": (4, 4, 64), "grouped64": (16, 2, 64), "grouped": (32, 8, 128)}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rotary_case(name, heads, dtype, B, L, layout, rot, scaling, far, packed, inverse):
    c = {"op": "rotary", "heads": heads, "dtype": dtype, "B": B, "L": L, "layout": layout, "rot": rot,
         "scaling": scaling, "far": far, "packed": packed, "inverse": inverse}
    return dict(c, name=name) if name else c


def _attention_case(name, heads, dtype, docs, q, kv, mix, block, prefix, cap, bias, middle, pad):
    c = {"op": "attention", "heads": heads, "dtype": dtype, "docs": docs, "q": q, "kv": kv, "mix": mix, "block": block,
         "prefix": prefix, "cap": cap, "bias": bias, "middle": middle, "pad": pad}
    return dict(c, name=name) if name else c


def _sample_case(name, dtype, R, V, std, temperature, top_k, top_p, min_p):
    c = {"op": "sample", "dtype": dtype, "R": R, "V": V, "std": std, "temperature": temperature, "top_k": top_k,
         "top_p": top_p, "min_p": min_p}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token of sixteen requests at positions of their own: launch latency
        _rotary_case("rotary_token", "dream", "bf16", 16, 1, "half", 128, "none", 8448, False, False),
        # a long prompt's queries and keys, positions scaled by parts beyond the trained length: bandwidth
        _rotary_case("rotary_long", "dream", "bf16", 1, 8448, "half", 128, "parts", 131072, False, False),
        # half of each head, interleaved, float32, read out of a packed projection at an odd length, undone again
        _rotary_case("rotary_partial", "llada", "f32", 4, 1023, "interleaved", 64, "linear", 40000, True, True),
        # one token of sixteen requests over caches of unlike lengths
        _attention_case("attention_token", "dream", "bf16", 16, 1, 8448, 1, 1, 0, 0.0, False, False, 0),
        # the block rows of a cached denoising step, batch 8: 32 queries in the middle of 1024 positions
        _attention_case("attention_block", "llada", "bf16", 8, 32, 1024, 0, 0, 0, 0.0, False, True, 0),
        # prompts of unlike lengths packed without padding, every position visible within its prompt, scores capped
        _attention_case("attention_packed", "llada", "bf16", 8, 1056, 0, 2, 0, 0, 50.0, False, False, 37),
        # one long sequence whose prompt is visible to all and whose blocks of 32 see what is to their left
        _attention_case("attention_prefix", "dream", "bf16", 1, 8448, 0, 0, 32, 512, 0.0, False, False, 0),
        # the tiny float32 model's heads, ragged, causal with distance biases: latency
        _attention_case("attention_bias", "tiny", "f32", 4, 237, 0, 3, 1, 0, 0.0, True, False, 5),
        # one row of one request: latency over a whole vocabulary
        _sample_case("sample_one", "f32", 1, 126464, 5.0, True, False, True, False),
        # a block of 32 rows, top-k then top-p
        _sample_case("sample_block", "f32", 32, 126464, 5.0, True, True, True, False),
        # batch 8 of 32 rows over flat logits, every control on
        _sample_case("sample_batch", "f32", 256, 152064, 1.2, True, True, True, True),
        # bf16 logits of an odd vocabulary, many of them equal
        _sample_case("sample_bf16", "bf16", 100, 3001, 3.0, True, False, True, True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "attention", "attention", "sample", "sample"])
    if op == "rotary":
        heads, dtype = rng.choice(list(HEADS)), rng.choice(["bf16", "bf16", "f32"])
        hd = HEADS[heads][2]
        B = _log(rng, 1, 16)
        L = _log(rng, 1, max(1, 4000 // B))
        return _rotary_case(None, heads, dtype, B, L, rng.choice(["half", "interleaved"]), rng.choice([hd, hd, hd // 2, hd // 4]),
                            rng.choice(["none", "linear", "parts"]), rng.choice([8448, 40000, 131072]), rng.random() < 0.5,
                            rng.random() < 0.3)
    if op == "attention":
        heads, dtype = rng.choice(list(HEADS)), rng.choice(["bf16", "bf16", "bf16", "f32"])
        kind = rng.choice(["token", "block", "packed"])
        block, prefix = rng.choice([(0, 0), (1, 0), (32, 0), (1, 100), (32, 70)])
        cap, bias = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.3
        mix, pad = rng.randrange(1, 1 << 20), rng.choice([0, 0, 3, 61])
        most = 1 if dtype == "bf16" else 2
        if kind == "token":
            return _attention_case(None, heads, dtype, _log(rng, 1, 24), rng.choice([1, 1, 1, 2, 4]), _log(rng, 20, 8448 // most), mix,
                                   block, prefix, cap, bias, False, pad)
        if kind == "block":
            return _attention_case(None, heads, dtype, _log(rng, 1, 8), rng.choice([16, 32, 33, 64]), _log(rng, 100, 3000 // most), mix,
                                   rng.choice([0, 32]), prefix, cap, bias, True, pad)
        docs = _log(rng, 1, 8)
        return _attention_case(None, heads, dtype, docs, _log(rng, 20, 5000 // most // docs), 0, mix, block, prefix, cap, bias, False, pad)
    R, V = _log(rng, 1, 256), _log(rng, 500, 152064)
    return _sample_case(None, rng.choice(["f32", "f32", "bf16"]), R, V, rng.choice([1.2, 3.0, 5.0]), rng.random() < 0.8,
                        rng.random() < 0.5, rng.random() < 0.6, rng.random() < 0.4)


# ---------------------------------------------------------------- sizes that a case stands for
def _lengths(c):
    """Query and key lengths of each document, and the position of its first query."""
    rng = random.Random(c["mix"])
    spread = lambda n: n if not c["mix"] else max(1, int(n * rng.uniform(0.3, 1.0)))  # noqa: E731
    q, kv, pos = [], [], []
    for _ in range(c["docs"]):
        if c["kv"]:
            kv.append(spread(c["kv"]))
            q.append(min(c["q"], kv[-1]))
            pos.append((kv[-1] - q[-1]) // 2 // 32 * 32 if c["middle"] else kv[-1] - q[-1])
        else:
            q.append(spread(c["q"]))
            kv.append(q[-1])
            pos.append(0)
    return q, kv, pos


def _visible(c, pos, n, kv):
    """Key counts that the n queries from position pos on see."""
    if not c["block"]:
        return n * kv
    return sum(min(kv, max(c["prefix"], ((pos + i) // c["block"] + 1) * c["block"])) for i in range(n))


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rotary":
        Hq, Hkv, hd = HEADS[c["heads"]]
        n = c["B"] * c["L"]
        return {"bytes": 2.0 * n * (Hq + Hkv) * hd * size + 4.0 * n, "flops": 3.0 * n * (Hq + Hkv) * c["rot"]}
    if c["op"] == "attention":
        Hq, Hkv, hd = HEADS[c["heads"]]
        q, kv, pos = _lengths(c)
        pairs = sum(_visible(c, p, a, b) for a, b, p in zip(q, kv, pos))
        return {"bytes": 2.0 * size * hd * (Hq * sum(q) + Hkv * sum(kv)), "flops": 4.0 * Hq * hd * pairs}
    return {"bytes": float(c["R"] * (c["V"] * size + 32)), "flops": 4.0 * c["R"] * c["V"]}


# ---------------------------------------------------------------- inputs
def _generator(seed, salt):
    return torch.Generator(device="cuda").manual_seed((seed * 7919 + salt) % (1 << 31))


def _normal(shape, seed, salt, std, dtype):
    return (torch.randn(shape, generator=_generator(seed, salt), device="cuda") * std).to(dtype)


def _uniform(shape, seed, salt, lo, hi):
    return torch.rand(shape, generator=_generator(seed, salt), device="cuda") * (hi - lo) + lo


def _rotary_cfg(c):
    """Arguments of the rotation: rates base^(-2j/rot), scaled linearly or by parts."""
    cfg = {"head_dim": HEADS[c["heads"]][2], "rot_dim": c["rot"], "interleaved": c["layout"] == "interleaved", "base": 1e6}
    if c["scaling"] == "linear":
        cfg.update(scaling="linear", factor=4.0)
    elif c["scaling"] == "parts":
        cfg.update(scaling="parts", factor=16.0, orig_len=8192, low=1.0, high=32.0, gain=0.1 * math.log(16.0) + 1.0)
    return cfg


def _rotary_inputs(c, seed):
    Hq, Hkv, hd = HEADS[c["heads"]]
    B, L, dt = c["B"], c["L"], TYPES[c["dtype"]]
    x = _normal((B, L, Hq + 2 * Hkv, hd), seed, 1, 1.3, dt)
    q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv]
    if not c["packed"]:
        q, k = q.contiguous(), k.contiguous()
    first = torch.randint(0, max(1, c["far"] - L), (B, 1), generator=_generator(seed, 2), device="cuda")
    return q, k, (first + torch.arange(L, device="cuda")).to(torch.int32)


def _attention_inputs(c, seed):
    Hq, Hkv, hd = HEADS[c["heads"]]
    ql, kl, pos = _lengths(c)
    dt, n, m = TYPES[c["dtype"]], sum(ql) + c["pad"], sum(kl) + c["pad"]
    s = {"q": _normal((n, Hq, hd), seed, 3, 1.3, dt), "k": _normal((m, Hkv, hd), seed, 4, 1.3, dt),
         "v": _normal((m, Hkv, hd), seed, 5, 1.3, dt), "out": _normal((n, Hq, hd), seed, 6, 1.0, dt)}
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s["q_len"], s["kv_len"], s["q_pos"] = ints(ql), ints(kl), ints(pos)
    s["q_start"] = ints([sum(ql[:i]) for i in range(len(ql))])
    s["kv_start"] = ints([sum(kl[:i]) for i in range(len(kl))])
    s["prefix"] = ints([c["prefix"]] * len(ql)) if c["prefix"] else None
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device="cuda") if c["bias"] else None
    return s


def _sample_inputs(c, seed):
    R, V = c["R"], c["V"]
    s = {"logits": _normal((R, V), seed, 7, c["std"], TYPES[c["dtype"]]), "u": _uniform((R,), seed, 8, 0.0, 1.0).clamp_(max=1 - 2.0 ** -24)}
    s["temperature"] = _uniform((R,), seed, 9, 0.3, 1.5) if c["temperature"] else None
    s["top_k"] = torch.randint(1, min(V, 2000), (R,), generator=_generator(seed, 10), device="cuda").to(torch.int32) if c["top_k"] else None
    s["top_p"] = _uniform((R,), seed, 11, 0.5, 1.0) if c["top_p"] else None
    s["min_p"] = _uniform((R,), seed, 12, 0.0, 0.1) if c["min_p"] else None
    if c["temperature"] and R > 4:  # a greedy request among the sampled ones
        s["temperature"][R // 2] = 0.0
    return s


def prepare(case, seed):
    c = case
    s = {"c": c}
    if c["op"] == "rotary":
        s["cfg"] = _rotary_cfg(c)
        s["q"], s["k"], s["pos"] = _rotary_inputs(c, seed)
    elif c["op"] == "attention":
        s.update(_attention_inputs(c, seed))
        s["max_q"], s["max_kv"] = max(_lengths(c)[0]), max(_lengths(c)[1])
    else:
        s.update(_sample_inputs(c, seed))
        s["mask_id"] = c["V"] - 1
    return s


# ---------------------------------------------------------------- plain forms
def _rates(cfg, device):
    """Angle per position of each pair, in 64 bits."""
    rot = cfg["rot_dim"]
    f = cfg["base"] ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=device) / rot)
    if cfg.get("scaling") == "linear":
        f = f / cfg["factor"]
    elif cfg.get("scaling") == "parts":
        turns = cfg["orig_len"] * f / (2 * math.pi)
        keep = ((turns - cfg["low"]) / (cfg["high"] - cfg["low"])).clamp(0, 1)
        f = f / cfg["factor"] * (1 - keep) + f * keep
    return f


def _rotate(x, cos, sin, rot, interleaved):
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([r, y[..., rot:]], -1).to(x.dtype)


def _plain_rotary(s):
    cfg = s["cfg"]
    ang = s["pos"].double()[..., None] * _rates(cfg, "cuda")
    gain = cfg.get("gain", 1.0)
    cos, sin = (torch.cos(ang) * gain).float()[:, :, None], (torch.sin(ang) * gain).float()[:, :, None]
    if s["c"]["inverse"]:
        sin = -sin
    return [_rotate(x, cos, sin, cfg["rot_dim"], cfg["interleaved"]) for x in (s["q"], s["k"])]


def _plain_attention(s):
    c = s["c"]
    Hq, Hkv, hd = HEADS[c["heads"]]
    n, m, g = s["q"].shape[0], s["k"].shape[0], Hq // Hkv
    row, col = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
    d = torch.searchsorted(s["q_start"], row.int(), right=True) - 1
    at = row - s["q_start"][d]
    covered = at < s["q_len"][d]
    pos = s["q_pos"][d] + at
    key = col[None, :] - s["kv_start"][d][:, None]
    sees = (key >= 0) & (key < s["kv_len"][d][:, None]) & covered[:, None]
    if c["block"]:
        end = (torch.div(pos, c["block"], rounding_mode="floor") + 1) * c["block"]
        if s["prefix"] is not None:
            end = torch.maximum(end, s["prefix"][d])
        sees &= key < end[:, None]
    q = s["q"].float().view(n, Hkv, g, hd).permute(1, 2, 0, 3).reshape(Hkv, g * n, hd)
    k, v = s["k"].float().transpose(0, 1).contiguous(), s["v"].float().transpose(0, 1).contiguous()
    x = (q @ k.transpose(1, 2).contiguous()).view(Hkv, g, n, m)
    x *= 1.0 / math.sqrt(hd)
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    if s["slopes"] is not None:
        x -= s["slopes"].view(Hkv, g, 1, 1) * (pos[:, None] - key).abs().float()
    x.masked_fill_(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    y = (x.view(Hkv, g * n, m) @ v).view(Hkv, g, n, hd) / torch.where(total == 0, torch.ones_like(total), total)
    y = y.permute(2, 0, 1, 3).reshape(n, Hq, hd).to(s["out"].dtype)
    s["out"].copy_(torch.where(covered[:, None, None], y, s["out"]))
    return s["out"]


def _plain_sample(s):
    x = s["logits"].double()
    R, V = x.shape
    x[:, s["mask_id"]] = -math.inf
    greedy = torch.zeros((R, 1), dtype=torch.bool, device="cuda")
    z = x
    if s["temperature"] is not None:
        t = s["temperature"].double()[:, None]
        greedy = t <= 0
        z = x / torch.where(greedy, torch.ones_like(t), t)
    w = torch.exp(z - z.amax(-1, keepdim=True))
    ranked, order = torch.sort(x, dim=-1, descending=True, stable=True)  # equal logits: lower index first
    del ranked
    wr = w.gather(1, order)
    rank = torch.arange(V, device="cuda")[None, :]
    keep = wr > 0
    if s["top_k"] is not None:
        keep &= rank < s["top_k"][:, None]
    if s["top_p"] is not None:
        c = torch.cumsum(wr * keep, -1)
        before = torch.cat([torch.zeros_like(c[:, :1]), c[:, :-1]], -1)
        keep &= (before < s["top_p"].double()[:, None] * c[:, -1:]) | (rank == 0)
    if s["min_p"] is not None:
        keep &= wr >= s["min_p"].double()[:, None]
    keep = torch.where(greedy, rank == 0, keep)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    c = torch.cumsum(w * kept, -1)
    token = (c <= s["u"].double()[:, None] * c[:, -1:]).sum(-1)
    last = torch.where(kept, rank, torch.zeros_like(rank)).amax(-1)
    token = torch.minimum(token, last)[:, None]
    e = torch.exp(x - x.amax(-1, keepdim=True))
    conf = e.gather(1, token) / e.sum(-1, keepdim=True)
    prob = w.gather(1, token) / c[:, -1:]
    return {"token": token[:, 0].int(), "conf": conf[:, 0].float(), "prob": prob[:, 0].float()}


# ---------------------------------------------------------------- one pass
def run(state):
    s, c = state, state["c"]
    if not own:
        return {"rotary": _plain_rotary, "attention": _plain_attention, "sample": _plain_sample}[c["op"]](s)
    from paper_2608_22646_amd import binding
    if c["op"] == "rotary":
        return list(binding.rotary(binding.Rotary(**s["cfg"]), s["q"], s["k"], pos=s["pos"], inverse=c["inverse"]))
    if c["op"] == "attention":
        docs = binding.Docs(s["q_start"], s["q_len"], s["kv_start"], s["kv_len"], s["max_q"], s["max_kv"], q_pos=s["q_pos"],
                            prefix=s["prefix"])
        return binding.attention(s["q"], s["k"], s["v"], docs, block=c["block"], cap=c["cap"], slopes=s["slopes"], out=s["out"])
    token, conf, prob = binding.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                       min_p=s["min_p"], mask_id=s["mask_id"])
    return {"token": token, "conf": conf, "prob": prob}


# ---------------------------------------------------------------- the same in 64 bits
def _exact_rotary(c, seed):
    q, k, pos = _rotary_inputs(c, seed)
    rot, scaling = c["rot"], c["scaling"]
    f = [1e6 ** (-2.0 * j / rot) for j in range(rot // 2)]
    gain = 1.0
    if scaling == "linear":
        f = [x / 4.0 for x in f]
    if scaling == "parts":
        gain = 1.0 + 0.1 * math.log(16.0)
        part = [min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1.0) / 31.0)) for x in f]
        f = [(1 - p) * x / 16.0 + p * x for x, p in zip(f, part)]
    turn = torch.polar(torch.full((), gain, dtype=torch.float64, device="cuda"),
                       pos.double()[:, :, None, None] * torch.tensor(f, dtype=torch.float64, device="cuda") * (-1.0 if c["inverse"] else 1.0))
    out = []
    for x in (q.double(), k.double()):
        y = x.clone()
        if c["layout"] == "interleaved":
            z = torch.view_as_complex(x[..., :rot].reshape(*x.shape[:-1], rot // 2, 2).contiguous()) * turn
            y[..., :rot] = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
            y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
        out.append(y)
    return out


def _exact_attention(c, seed):
    Hq, Hkv, hd = HEADS[c["heads"]]
    s = _attention_inputs(c, seed)
    ql, kl, pos = _lengths(c)
    out = s["out"].double()
    q0 = k0 = 0
    for a, b, p in zip(ql, kl, pos):
        i = torch.arange(p, p + a, device="cuda")[:, None]
        j = torch.arange(b, device="cuda")[None, :]
        hidden = None
        if c["block"]:
            hidden = (j >= c["prefix"]) & (j // c["block"] > i // c["block"])
        for h in range(Hq):
            x = s["q"][q0:q0 + a, h].double() @ s["k"][k0:k0 + b, h // (Hq // Hkv)].double().T.contiguous() / math.sqrt(hd)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if c["bias"]:
                x = x - 2.0 ** (-8.0 * (h + 1) / Hq) * (i - j).abs()
            if hidden is not None:
                x[hidden] = -math.inf
            out[q0:q0 + a, h] = torch.softmax(x, -1) @ s["v"][k0:k0 + b, h // (Hq // Hkv)].double().contiguous()
        q0, k0 = q0 + a, k0 + b
    return out


def _exact_sample(c, seed):
    s = _sample_inputs(c, seed)
    R, V = c["R"], c["V"]
    token, conf, prob = [], [], []
    for r in range(R):
        x = s["logits"][r, :V - 1].double()  # the mask token is the last one
        t = 1.0 if s["temperature"] is None else float(s["temperature"][r])
        order = torch.argsort(x, descending=True, stable=True)
        if t <= 0:
            pick, share = order[0], torch.ones((), dtype=torch.float64, device="cuda")
        else:
            p = torch.softmax(x / t, -1)
            if s["top_k"] is not None:
                order = order[:int(s["top_k"][r])]
            if s["top_p"] is not None:
                mass = torch.cumsum(p[order], 0)
                order = order[:1 + int((mass[:-1] < float(s["top_p"][r]) * mass[-1]).sum())]
            if s["min_p"] is not None:
                order = order[p[order] >= float(s["min_p"][r]) * p.max()]
            index = torch.sort(order).values
            mass = torch.cumsum(p[index], 0)
            pick = index[min(int((mass <= float(s["u"][r]) * mass[-1]).sum()), len(index) - 1)]
            share = p[pick] / mass[-1]
        token.append(pick)
        conf.append(torch.softmax(x, -1)[pick])
        prob.append(share)
    return {"token": torch.stack(token).int(), "conf": torch.stack(conf), "prob": torch.stack(prob)}


def exact(case, seed):
    return {"rotary": _exact_rotary, "attention": _exact_attention, "sample": _exact_sample}[case["op"]](case, seed)
