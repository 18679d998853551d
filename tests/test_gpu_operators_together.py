"""Stand-alone operators as they are used together, beside the model's own path:
rotary and attention on a layer's normed input against what the layer leaves, a
cache that grows by a token a step, and a decode whose tokens are sampled."""
import math

import numpy as np
import pytest
import torch

from gpu_stages import ws_view
from helpers import assert_bf16_flips, assert_state_equal, replay, say, to_np
from oracle import forward as of
from oracle import operators as oo
from paper_2608_22646_amd import binding as B
from paper_2608_22646_amd import synth

pytestmark = pytest.mark.gpu

SMALL = synth.ModelConfig("together-bf16", n_layers=1, d_model=512, n_heads=4, n_kv_heads=2, head_dim=128, d_ff=768,
                          vocab=3001, rope_base=1e4, dtype="bf16", lm_head_std=5 / math.sqrt(512))


def randn(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).cuda()


def test_rotary_and_attention_are_a_layers(gpu_lib):
    """q and k may differ from the layer's by bf16 flips; attention of the layer's own q, k and v
    by what both round: probabilities (2^-8 and, in half, 2^-11, of their sum over |v|), float32
    sums (2^-16 of it) and the result."""
    cfg, Bn, L = SMALL, 2, 100
    H, Hkv, hd, M = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, Bn * L
    w = synth.make_weights(cfg, "cuda")
    model = B.Model(cfg, w)
    ws = model.workspace(Bn, L, 0)
    x = synth.make_ints((Bn, L), 5, 0, cfg.vocab).cuda()
    say("operators against a layer")
    model.embed(x, ws)
    model.layer(0, 0, Bn, L, ws)
    torch.cuda.synchronize()
    lay = model.layout(Bn, L, 0)
    a = to_np(ws_view(ws, lay.a_attn, torch.bfloat16, (M, cfg.d_model)), np.float64)
    wq, wk, wv = (to_np(t, np.float64) for t in w[2:5])
    proj = lambda m, n: torch.from_numpy(of._matmul(a, m, "bf16")).float().view(Bn, L, n, hd).cuda()  # noqa: E731
    q, k = B.rotary(B.Rotary(hd, base=cfg.rope_base), proj(wq, H), proj(wk, Hkv))
    q, k, v = q.bfloat16(), k.bfloat16(), proj(wv, Hkv).bfloat16()
    q_l = ws_view(ws, lay.q, torch.bfloat16, (Bn, H, L, hd)).permute(0, 2, 1, 3)
    k_l = ws_view(ws, lay.k, torch.bfloat16, (Bn, Hkv, L, hd)).permute(0, 2, 1, 3)
    v_l = ws_view(ws, lay.vt, torch.float16, (Bn, Hkv, hd, L)).permute(0, 3, 1, 2).bfloat16().contiguous()
    for name, g, r in (("q", q, q_l), ("k", k, k_l), ("v", v, v_l)):
        assert_bf16_flips(to_np(r, np.float64), to_np(g, np.float64), name)

    got = to_np(B.attention(q_l, k_l, v_l).reshape(M, H * hd), np.float64)
    layer = to_np(ws_view(ws, lay.attn, torch.bfloat16, (M, H * hd)), np.float64)
    mass = np.concatenate([oo.attention(to_np(q_l[b], np.float64), to_np(k_l[b], np.float64), to_np(v_l[b], np.float64), 0, 0, 0,
                                        1 / math.sqrt(hd), 0.0, None)[1] for b in range(Bn)]).reshape(M, H * hd)
    tol = (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -16) * mass + 2.0 ** -8 * (np.abs(got) + np.abs(layer)) * 1.01
    assert (np.abs(got - layer) <= tol).all(), (np.abs(got - layer) / tol).max()


class Cache:
    """A left-padded batch whose sequence d begins at column start[d] of its slab."""

    def __init__(self, start, columns, heads, seed):
        self.Hq, self.Hkv, self.hd = heads
        self.D = len(start)
        self.k, self.v = (torch.full((self.D, columns, self.Hkv, self.hd), float("nan"), device="cuda") for _ in "kv")
        self.start = torch.tensor(start, dtype=torch.int32, device="cuda")
        self.n = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.rope = B.Rotary(self.hd, base=1e4, scaling="linear", factor=2.0)
        self.seen = []   # (q, k, v) as they came, for the oracle
        self.seed = seed

    def new(self, cols):
        out = [randn((self.D, cols, h, self.hd), self.seed + i, 1.3) for i, h in enumerate((self.Hq, self.Hkv, self.Hkv))]
        self.seed += 3
        self.seen.append(out)
        return out

    def append(self, q, k, v, at, lens, ws):
        """Columns at .. of the batch: rotates q, stores the rotated k and v, attends block-causally."""
        cols = q.shape[1]
        pos = torch.arange(at, at + cols, dtype=torch.int32, device="cuda")[None] - self.start[:, None]
        qr, _ = B.rotary(self.rope, q, k, pos=pos.contiguous(), k_out=self.k[:, at:at + cols])
        self.v[:, at:at + cols] = v
        docs = B.Docs(kv_start=self.start, kv_len=lens, max_q=cols, max_kv=self.k.shape[1])
        return B.attention(qr, self.k, self.v, docs, block=1, ws=ws)

    def reference(self, at, cols):
        """(output, tolerance) [D, cols, Hq, hd] of the columns at .. by the oracle."""
        q, k, v = (torch.cat([s[i] for s in self.seen], 1) for i in range(3))
        u, sc = 2.0 ** -24, float(np.float32(1 / math.sqrt(self.hd)))
        ref, tol, rates = [], [], oo.rotary_rates(self.hd, 1e4, "linear", 2.0)
        pairs = lambda x: np.hypot(x[..., :self.hd // 2], x[..., self.hd // 2:])  # noqa: E731
        for d in range(self.D):
            s = int(self.start[d])
            rot = lambda x, p: oo.rotary(to_np(x, np.float64)[None], p[None], rates)[0]  # noqa: E731
            n = at + cols - s
            qr, kr = rot(q[d, at:at + cols], np.arange(at - s, n)), rot(k[d, s:at + cols], np.arange(n))
            o, mass, top, dot = oo.attention(qr, kr, to_np(v[d, s:at + cols], np.float64), at - s, 1, 0, sc, 0.0, None)
            # as for attention alone, and for the rotated operands: an element is off by 4 u of |a| + |b| of its
            # pair, so a score by 16 u of the sum of its pairs' |q| |k|
            nq, nk = pairs(qr), pairs(kr)
            turned = np.stack([(nq[:, h] @ nk[:, h // (self.Hq // self.Hkv)].T).max(1) for h in range(self.Hq)], 1)
            e = u * ((self.hd + 8) * sc * dot + 8 * top + 16 * sc * turned)
            ref.append(o)
            tol.append((2 * e + (8 + n) * u)[:, :, None] * mass * 1.01 + u * np.abs(o) * 1.01)
        return np.stack(ref), np.stack(tol)


def test_a_cache_that_grows(gpu_lib):
    """A left-padded batch: 40 columns at once, then one a step."""
    c = Cache([0, 5, 17], 700, (4, 2, 64), 100)
    at = 0
    for cols in (40, 1, 1, 3, 1, 530, 1):
        say(f"cache: columns {at} .. {at + cols - 1}")
        q, k, v = c.new(cols)
        out = to_np(c.append(q, k, v, at, at + cols - c.start, None), np.float64)
        ref, tol = c.reference(at, cols)
        for d, s in enumerate((0, 5, 17)):
            real = slice(max(0, s - at), None)     # (columns before a sequence's first hold nothing of it)
            assert (np.abs(out[d, real] - ref[d, real]) <= tol[d, real]).all(), f"sequence {d}, column {at}"
        at += cols


def test_a_step_in_a_graph(gpu_lib):
    """Rotary, the store into the cache, attention and sampling captured as one graph, and a second one of
    another step over the same workspaces: replays in turn, on changed inputs, give what eager calls give."""
    c = Cache([3, 0, 9], 600, (8, 2, 64), 300)
    q, k, v = c.new(400)
    c.append(q, k, v, 0, 400 - c.start, None)
    u = torch.rand(3, generator=torch.Generator().manual_seed(1)).cuda()
    temp, top_p = torch.full((3,), 0.7, device="cuda"), torch.full((3,), 0.9, device="cuda")
    lens = {at: (at + 1 - c.start).contiguous() for at in (400, 401)}
    one = c.new(1)
    docs = B.Docs(kv_start=c.start, kv_len=lens[400], max_q=1, max_kv=600)
    aws = B.device_buffer(max(B.attention_workspace_size(one[0], c.k, c.v, docs), 256))
    sws = B.device_buffer(B.sample_workspace_size(3, 8 * 64))

    def step(at):
        o = c.append(*one, at, lens[at], aws)
        return (o, *B.sample(o.view(3, -1), u, temp, top_p=top_p, ws=sws))

    graphs, outs = {}, {}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for at in (400, 401):
            step(at)
            graphs[at] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[at], stream=side):
                outs[at] = step(at)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for i in range(3):
        say(f"replays {i}")
        for n, t in enumerate(one):
            t.copy_(randn(t.shape, 900 + 10 * i + n, 1.3))
        u.copy_(torch.rand(3, generator=torch.Generator().manual_seed(50 + i)))
        want = {at: [t.clone() for t in step(at)] for at in (400, 401)}
        c.k[:, 400:402] = float("nan")
        torch.cuda.synchronize()
        for at in (400, 401):
            graphs[at].replay()
        torch.cuda.synchronize()
        for at in (400, 401):
            for g, r in zip(outs[at], want[at]):
                assert torch.equal(g, r)


@pytest.mark.parametrize("gating", [True, False])
def test_a_sampled_decode(gpu_lib, gating):
    """forward, sample in place of the argmax, commit: tokens by the oracle on the forward's logits, decisions
    by the oracle's controller on the sampled (confidence, token)."""
    cfg, Bn, P, G = synth.TINY, 2, 16, 64
    model = B.Model(cfg, synth.make_weights(cfg, "cuda"))
    ctl = B.Controller.gating(gating)
    bl, T, nb = ctl.block_len, ctl.T, 64 // ctl.block_len
    prompt = synth.make_ints((Bn, P), 3, 0, cfg.mask_id)
    st = B.DecodeState(Bn, P, G)
    B.state_init(cfg.mask_id, prompt.cuda(), G, st)
    ws = model.workspace(Bn, P + G, bl)
    temp = torch.tensor([0.6, 1.1]).repeat_interleave(bl).cuda()
    top_p, top_k = torch.full((Bn * bl,), 0.95).cuda(), torch.full((Bn * bl,), 300, dtype=torch.int32).cuda()
    confs, args = np.zeros((nb, T, Bn, bl), np.float32), np.zeros((nb, T, Bn, bl), np.int64)
    flag, forwards, greedy = torch.zeros(1, dtype=torch.int32, device="cuda"), [], 0
    for blk in range(nb):
        for t in range(T):
            say(f"sampled decode: block {blk} step {t}")
            _, arg, lg = model.forward(st.x, P + blk * bl, bl, ws, logits=True)
            u = torch.rand(Bn * bl, generator=torch.Generator().manual_seed(blk * T + t))
            token, conf, _ = B.sample(lg.view(Bn * bl, -1), u.cuda(), temp, top_k, top_p, mask_id=cfg.mask_id)
            B.commit(ctl, st, conf.view(Bn, bl), token.view(Bn, bl), blk, t, cfg.mask_id, flag)
            confs[blk, t], args[blk, t] = conf.view(Bn, bl).cpu().numpy(), token.view(Bn, bl).cpu().numpy()
            greedy += int((token == arg.view(-1)).sum())
            lgn, tn = to_np(lg.view(Bn * bl, -1), np.float64), to_np(temp, np.float64)
            for r in range(0, Bn * bl, 5):
                assert int(token[r]) == oo.sample(lgn[r], float(u[r]), tn[r], 300, float(np.float32(0.95)), 0.0, cfg.mask_id)[0]
            if int(flag.item()):
                break
        forwards.append(t + 1)
    assert 0 < greedy < sum(forwards) * Bn * bl
    ref = replay(confs, args, prompt.numpy(), G, cfg.mask_id, ctl)
    assert_state_equal(st, forwards, ref)
