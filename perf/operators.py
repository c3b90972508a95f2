"""Operators around a grafted cache, for timing and for comparing outputs.

Four operators and how a program uses them:

``rope``    encode queries and keys at their positions in one of the rotary forms
            (``fcg_rope_apply``), or take a gradient back through it
``append``  place a call's keys and values into a cache, the rotation applied on the
            way (``fcg_append``); a pass writes the same positions again, as a retry
            of a patched span does
``graft``   stitch library segments of another rotary form into a cache
            (``fcg_graft_rope``), after a reset of the sequences
``attend``  attention of many sequences over one shared prefix and their own tokens
            (``fcg_prefix_attend``)

Fields of a case: ``hq``, ``hkv``, ``d``, ``dtype``, ``layers``; the rotary form
(``layout`` half or pairs, ``rot`` rotated dimensions, ``theta``, ``scale`` its long
context scaling with ``factor``, ``m`` the factor on the encoded vectors); ``page`` (0
contiguous, 16 paged); ``seqs`` sequences of ``tok_min`` .. ``tok_max`` tokens a call;
``far`` the largest position; ``plan`` seed of lengths and positions.  ``rope``:
``fused`` q and k are slices of one projection output, ``grad`` the backward pass.
``graft``: ``segs`` segments a sequence of ``seg_min`` .. ``seg_max`` tokens out of
``lib``, after a ``prefix`` segment.  ``attend``: ``prefix`` shared positions, ``own_min``
.. ``own_max`` own positions before the call's last token.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BASE = dict(hq=32, hkv=8, d=128, dtype="bf16", layers=1, layout="half", rot=128, theta=1e6, scale="none", factor=1.0,
             m=1.0, page=0, seqs=1, tok_min=1, tok_max=1, far=4096, plan=1, fused=False, grad=False, segs=0, seg_min=0,
             seg_max=0, lib=0, prefix=0, own_min=0, own_max=0)
_PARTS = dict(scale="parts", factor=4.0, m=0.1 * math.log(4.0) + 1.0)      # by parts, to four times the trained length
_ORIG, _LO, _HI = 32768, 1.0, 32.0                                         # trained length and ramp of "parts"


def _case(name, op, *parts, **more):
    c = dict(_BASE, name=name, op=op)
    for p in parts:
        c.update(p)
    c.update(more)
    return c


def listed():
    return [
        # the smallest call: one decode token of a long-context task, queries and keys
        _case("rope-token", "rope", _PARTS, tok_min=1, tok_max=1, far=120000),
        # encoding the keys of a new library segment, all layers, in the layout of neighbouring pairs
        _case("rope-segment", "rope", layers=32, hq=0, layout="pairs", tok_min=713, tok_max=713, far=713),
        # training: the gradient of a prompt's queries and keys, fp32, 96 of 128 dimensions rotated, taken
        # from and with the strides of a fused projection
        _case("rope-grad-f32", "rope", hq=16, hkv=4, dtype="f32", rot=96, theta=1e4, tok_min=900, tok_max=1300,
              seqs=4, far=8192, fused=True, grad=True),
        # one decode step of a serving batch, one layer: a token for each of 64 paged tasks
        _case("append-step", "append", _PARTS, page=16, seqs=64, far=6000),
        # the patch tokens of one interactive task, all layers in one call, pairs layout, a quarter of the head
        _case("append-patch", "append", layers=32, layout="pairs", rot=32, tok_min=129, tok_max=129, far=4300),
        # prompts of a batch computed elsewhere and placed into the pages of eight layers
        _case("append-batch", "append", layers=8, page=16, seqs=32, tok_min=100, tok_max=600, far=700),
        # cache-stitching of one interactive task (system prompt + 6 functions) for a model whose rotary pairs
        # are neighbours
        _case("graft-pairs-7b", "graft", layers=32, layout="pairs", prefix=1024, segs=6, seg_min=200, seg_max=800,
              lib=32),
        # cache-stitching of a paged batch, half of each head rotated, positions interpolated to twice the length
        _case("graft-part-batch", "graft", layers=4, page=16, rot=64, theta=1e4, scale="linear", factor=2.0, seqs=16,
              segs=8, seg_min=500, seg_max=1000, lib=64),
        # the smallest attention: three candidates of a small fp32 model after ~450 shared tokens
        _case("attend-tiny-f32", "attend", hq=4, hkv=2, d=64, rot=64, dtype="f32", theta=1e4, page=16, seqs=3,
              prefix=449, own_min=1, own_max=40),
        # one decode step of 64 candidate programs over one stitched context of ~4.3K tokens
        _case("attend-step", "attend", page=16, seqs=64, prefix=4321, own_min=1, own_max=300),
        # drafts of four tokens for 32 tasks of a larger model (eight query heads a kv head) over ~22K shared tokens
        _case("attend-draft-34b", "attend", hq=64, page=16, seqs=32, prefix=22011, tok_min=4, tok_max=4, own_min=40,
              own_max=900),
        # the patch prompts of 32 tasks over a shared context: 64 tokens each
        _case("attend-patch", "attend", page=16, seqs=32, prefix=6007, tok_min=64, tok_max=64, own_min=64, own_max=300),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "graft", "attend", "attend"])
    c = dict(_BASE, op=op, plan=rng.randrange(1 << 20))
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (16, 4, 64), (8, 8, 64), (16, 1, 128), (4, 2, 64), (16, 8, 128)])
    c.update(hq=hq, hkv=hkv, d=d, theta=rng.choice([1e4, 1e6]))
    if rng.random() < 0.25:
        c["dtype"] = "f32"
    c["layout"] = rng.choice(["half", "pairs"])
    c["rot"] = rng.choice([d, d, d // 2, d // 4, d - 16, 16])
    c["scale"] = rng.choice(["none", "linear", "parts", "ntk"])
    if c["scale"] != "none":
        c["factor"] = rng.choice([2.0, 3.5, 8.0])
        c["m"] = rng.choice([1.0, 0.1 * math.log(c["factor"]) + 1.0])
    c["page"] = rng.choice([0, 16])
    c["far"] = _log_int(rng, 800, 30000)
    es = 4 if c["dtype"] == "f32" else 2
    if op in ("rope", "append"):
        c["seqs"] = _log_int(rng, 1, 64)
        c["layers"] = _log_int(rng, 1, 32)
        row = (hq + 2 * hkv) * d * es * 2 * c["layers"]
        top = max(1, min(2000, int(1e9 / (row * c["seqs"]))))
        c["tok_max"] = _log_int(rng, 1, top)
        c["tok_min"] = rng.randint(1, c["tok_max"])
        c["fused"] = rng.random() < 0.5
        if op == "rope":
            c["grad"] = rng.random() < 0.5
            c["far"] = _log_int(rng, 800, 1000000)
        else:   # the cache holds the tokens and where they start
            c["far"] = min(c["far"], max(c["tok_max"] + 1, int(3e8 / (hkv * d * es * 2 * c["layers"] * c["seqs"]))))
    elif op == "graft":
        c["seqs"] = _log_int(rng, 1, 16)
        c["segs"] = _log_int(rng, 1, 12)
        c["seg_max"] = _log_int(rng, 4, 1200)
        c["seg_min"] = rng.randint(1, c["seg_max"])
        c["lib"] = c["segs"] + rng.randrange(1, 24)
        c["prefix"] = rng.choice([0, _log_int(rng, 16, 1500)])
        tok = c["seqs"] * (c["prefix"] + c["segs"] * c["seg_max"]) + c["lib"] * c["seg_max"]
        c["layers"] = max(1, min(_log_int(rng, 1, 32), int(2e9 / (tok * hkv * d * es * 2))))
    else:
        c["seqs"] = _log_int(rng, 1, 64)
        c["tok_max"] = 1 if rng.random() < 0.5 else _log_int(rng, 2, 128)
        c["tok_min"] = rng.randint(1, c["tok_max"])
        c["prefix"] = _log_int(rng, 16, 22000) if rng.random() < 0.9 else 0
        c["own_max"] = _log_int(rng, c["tok_max"], max(c["tok_max"], 1000))
        c["own_min"] = rng.randint(c["tok_max"], c["own_max"])
        lim = 2e11 if es == 2 else 2e10
        while c["seqs"] > 1 and 4.0 * hq * d * c["seqs"] * c["tok_max"] * (c["prefix"] + c["own_max"]) > lim:
            c["seqs"] = (c["seqs"] + 1) // 2
    return c


# ------------------------------------------------------------------ sizes and positions (from the case alone)

def _freqs(c):
    """Frequencies of the rotary pairs, host float64."""
    r = c["rot"]
    theta = c["theta"] * c["factor"] ** (r / (r - 2)) if c["scale"] == "ntk" else c["theta"]
    w = [theta ** (-2.0 * i / r) for i in range(r // 2)]
    if c["scale"] == "linear":
        w = [x / c["factor"] for x in w]
    if c["scale"] == "parts":
        keep = [min(1.0, max(0.0, (_ORIG * x / (2 * math.pi) - _LO) / (_HI - _LO))) for x in w]
        w = [x * ((1 - k) / c["factor"] + k) for x, k in zip(w, keep)]
    return w


class _Plan:
    def __init__(self, c):
        rng = np.random.default_rng(c["plan"])
        S = c["seqs"]
        if c["op"] == "graft":
            self.lens = [int(x) for x in rng.integers(c["seg_min"], c["seg_max"], size=c["lib"], endpoint=True)]
            if c["prefix"]:
                self.lens.append(c["prefix"])
            self.off = np.concatenate([[0], np.cumsum(self.lens)]).astype(np.int64)
            self.seq, self.seg, self.dst, end = [], [], [], []
            for s in range(S):
                pos = 0
                picks = ([c["lib"]] if c["prefix"] else []) + [int(g) for g in rng.choice(c["lib"], c["segs"], False)]
                for g in picks:
                    self.seq.append(s), self.seg.append(g), self.dst.append(pos)
                    pos += self.lens[g]
                end.append(pos)
            self.T = -(-max(end) // 16) * 16
            tok = [(s, self.off[g] + j, dst + j, dst) for s, g, dst in zip(self.seq, self.seg, self.dst)
                   for j in range(self.lens[g])]
            self.t_seq, self.t_src, self.t_pos, self.t_delta = (np.array(x, dtype=np.int64) for x in zip(*tok))
        else:
            n = rng.integers(c["tok_min"], c["tok_max"], size=S, endpoint=True)
            if c["op"] == "attend":
                own_len = np.maximum(n, rng.integers(c["own_min"], c["own_max"], size=S, endpoint=True))
                self.own_len = own_len.astype(np.int64)
                start = c["prefix"] + own_len - n
                self.T = -(-(c["prefix"] + int(own_len.max())) // 16) * 16
            else:
                start = rng.integers(0, np.maximum(1, c["far"] - n), size=S, endpoint=True)
                self.T = -(-int((start + n).max()) // 16) * 16
            self.n = n.astype(np.int64)
            self.t_seq = np.repeat(np.arange(S), n)
            self.t_pos = np.concatenate([np.arange(a, a + k) for a, k in zip(start, n)]).astype(np.int64)
        # pages of the tokens, numbered in (sequence, page) order as one call maps them
        key = self.t_seq.astype(np.int64) * (self.T // 16) + self.t_pos // 16
        self.page_key, page = np.unique(key, return_inverse=True)
        self.slot = page.astype(np.int64) * 16 + self.t_pos % 16


class _Values:
    def __init__(self, c, seed):
        self.dt = _DT[c["dtype"]]
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def __call__(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.g, device="cuda") * scale).to(self.dt)


def _tensors(c, seed):
    """The values of a case, drawn in a fixed order."""
    p, vals = _Plan(c), _Values(c, seed)
    L, d, hq, hkv = c["layers"], c["d"], c["hq"], c["hkv"]
    t = {}
    if c["op"] in ("rope", "append"):
        n = len(p.t_pos)
        if c["fused"]:      # slices of one projection output [L][n][hq + 2 hkv][d]
            x = vals(L, n, hq + 2 * hkv, d)
            t["q"], t["k"], t["v"] = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        else:
            t["q"], t["k"], t["v"] = vals(L, n, hq, d), vals(L, n, hkv, d), vals(L, n, hkv, d)
    elif c["op"] == "graft":
        t["k"], t["v"] = vals(L, hkv, int(p.off[-1]), d, scale=0.5), vals(L, hkv, int(p.off[-1]), d, scale=0.5)
    else:
        own_max = int(p.own_len.max())
        t["q"] = vals(len(p.t_pos), hq, d)
        t["pk"], t["pv"] = vals(hkv, c["prefix"], d), vals(hkv, c["prefix"], d)
        t["k"], t["v"] = vals(c["seqs"], hkv, own_max, d), vals(c["seqs"], hkv, own_max, d)
    return p, t


# ------------------------------------------------------------------ what a program has before the call

class _Memory:
    """Device memory of a cache, for torch.as_tensor; keeps the handles it belongs to."""

    def __init__(self, ptr, n, es, keep):
        self.keep = keep
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": "<f4" if es == 4 else "<i2", "data": (ptr, False),
                                         "version": 2}


def _cache_memory(fcg, cache, shape, dt, keep):
    es = 4 if dt == torch.float32 else 2
    out = []
    for ptr in fcg.fcg_cache_device_ptrs(cache, 0):
        m = torch.as_tensor(_Memory(ptr, math.prod(shape), es, keep), device="cuda")
        out.append((m if es == 4 else m.view(dt)).view(shape))
    return out


def _make_rope(fcg, c):
    kind = {"none": fcg.FCG_ROPE_PLAIN, "linear": fcg.FCG_ROPE_LINEAR, "ntk": fcg.FCG_ROPE_NTK,
            "parts": fcg.FCG_ROPE_PARTS}[c["scale"]]
    layout = fcg.FCG_ROPE_HALF if c["layout"] == "half" else fcg.FCG_ROPE_PAIRS
    return fcg.fcg_rope_create(c["rot"], c["theta"], layout=layout, scaling=kind, factor=c["factor"],
                               orig_tokens=_ORIG, low_turns=_LO, high_turns=_HI, attn_factor=c["m"])


def prepare(case, seed):
    c = case
    p, t = _tensors(c, seed)
    dt = _DT[c["dtype"]]
    dev = "cuda"
    L, S, hq, hkv, d = c["layers"], c["seqs"], c["hq"], c["hkv"], c["d"]
    st = {"case": c, "plan": p, **t}
    paged = c["page"] != 0
    if c["op"] in ("rope", "append"):
        st["q_out"] = torch.empty((L, len(p.t_pos), hq, d), dtype=dt, device=dev)
    if c["op"] == "rope":
        st["k_out"] = torch.empty((L, len(p.t_pos), hkv, d), dtype=dt, device=dev)
        st["pos"] = torch.as_tensor(p.t_pos, dtype=torch.int32, device=dev)
    n_pages = len(p.page_key)
    shape = (L, n_pages, hkv, 16, d) if paged else (L, S, hkv, p.T, d)
    if c["op"] == "attend":
        st["out"] = torch.empty((len(p.t_pos), hq, d), dtype=dt, device=dev)
        st["lse"] = torch.empty((len(p.t_pos), hq), dtype=torch.float32, device=dev)
    if not own:
        w = torch.tensor(_freqs(c), dtype=torch.float64, device=dev)
        st["w"] = w
        for key in ("t_seq", "t_pos", "t_src", "t_delta", "slot"):
            if hasattr(p, key):
                st[key] = torch.as_tensor(getattr(p, key), device=dev)
        if c["op"] in ("append", "graft"):
            st["K"], st["V"] = (torch.zeros(shape, dtype=dt, device=dev) for _ in range(2))
        if c["op"] == "attend":
            st["m"] = torch.as_tensor(p.n, device=dev)
            st["len"] = torch.as_tensor(p.own_len, device=dev)
            # row of each token in a [S][tok_max] arrangement
            st["row"] = torch.as_tensor(np.concatenate([np.arange(k) for k in p.n]), device=dev)
        return st
    from paper_2606_13097_amd import fcg
    st["fcg"] = fcg
    desc = fcg.model_desc(L, max(hq, hkv), hkv, d, c["theta"], c["dtype"])
    if c["op"] != "attend":
        st["rope"] = _make_rope(fcg, c)
    if c["op"] == "append":
        st["cache"] = fcg.fcg_cache_create(desc, S, p.T, c["page"], n_pages if paged else 0)
    elif c["op"] == "graft":
        st["lib"] = fcg.fcg_lib_create(desc, int(p.off[-1]), len(p.lens))
        for n in p.lens:
            fcg.fcg_lib_add_segment(st["lib"], n, 0)
        lk, lv = (torch.as_tensor(_Memory(ptr, t["k"].numel(), 4 if dt == torch.float32 else 2, st["lib"]), device=dev)
                  for ptr in fcg.fcg_lib_device_ptrs(st["lib"], 0))
        for mem, x in ((lk, t["k"]), (lv, t["v"])):
            (mem if dt == torch.float32 else mem.view(dt)).view(x.shape).copy_(x)
        st["cache"] = fcg.fcg_cache_create(desc, S, p.T, c["page"], n_pages if paged else 0)
    elif c["op"] == "attend":
        # the cache as a program leaves it: the prefix in sequence S, each task's own tokens after it
        sq = np.concatenate([np.full(c["prefix"], S)] + [np.full(n, s) for s, n in enumerate(p.own_len)])
        ps = np.concatenate([np.arange(c["prefix"])] + [np.arange(c["prefix"], c["prefix"] + n) for n in p.own_len])
        total = sum(-(-(c["prefix"] + n) // 16) for n in p.own_len) + -(-max(c["prefix"], 1) // 16)
        st["cache"] = cache = fcg.fcg_cache_create(desc, S + 1, max(p.T, 16), c["page"], total if paged else 0)
        zero = torch.zeros((len(sq), hkv, d), dtype=dt, device=dev)
        fcg.fcg_append(cache, 0, sq, ps, zero, zero)
        shape = (1, total, hkv, 16, d) if paged else (1, S + 1, hkv, max(p.T, 16), d)
        for mem, pre, mine in zip(_cache_memory(fcg, cache, shape, dt, cache), (t["pk"], t["pv"]), (t["k"], t["v"])):
            for s in range(S + 1):
                x, at = (pre, 0) if s == S else (mine[s, :, :int(p.own_len[s])], c["prefix"])
                if not x.shape[1]:
                    continue
                if paged:
                    pt, _, _ = fcg.fcg_cache_export_layout(cache, s, 0)
                    pos = np.arange(at, at + x.shape[1])
                    page = torch.as_tensor(pt[pos // 16].astype(np.int64), device=dev)
                    mem[0][page, :, torch.as_tensor(pos % 16, device=dev)] = x.transpose(0, 1)
                else:
                    mem[0, s, :, at:at + x.shape[1]] = x
        st.update(pk=None, pv=None, k=None, v=None)
    if c["op"] in ("append", "graft"):
        st["K"], st["V"] = _cache_memory(fcg, st["cache"], shape, dt, st["cache"])
        st["K"].zero_(), st["V"].zero_()
    if c["op"] == "graft":
        st["g_seq"], st["g_seg"], st["g_dst"] = (np.array(x, dtype=np.int32) for x in (p.seq, p.seg, p.dst))
    else:
        st["h_seq"], st["h_pos"] = p.t_seq.astype(np.int32), p.t_pos.astype(np.int32)
    return st


# ------------------------------------------------------------------ one pass

def _turn(x, pos, c, w, sign=1.0, m=None):
    """The rotary turn of x [..., n, heads, d] at pos [n], in 32 bits with angles in 64, rounded once."""
    a = pos.to(torch.float64)[:, None] * w
    m = c["m"] if m is None else m
    cos, sin = (a.cos() * m).float()[:, None, :], (a.sin() * (m * sign)).float()[:, None, :]
    x32 = x.float()
    r = c["rot"]
    if c["layout"] == "half":
        xa, xb = x32[..., :r // 2], x32[..., r // 2:r]
        y = torch.cat([xa * cos - xb * sin, xb * cos + xa * sin, x32[..., r:]], dim=-1)
    else:
        xa, xb = x32[..., 0:r:2], x32[..., 1:r:2]
        y = torch.cat([torch.stack([xa * cos - xb * sin, xb * cos + xa * sin], dim=-1).flatten(-2), x32[..., r:]], -1)
    return y.to(x.dtype)


def _place(st, k, v):
    """k, v [L][n][hkv][d] into the cache memory at the tokens' places."""
    for mem, x in ((st["K"], k), (st["V"], v)):
        if st["case"]["page"]:
            mem[:, st["slot"] // 16, :, st["slot"] % 16] = x.transpose(0, 1)
        else:
            mem[:, st["t_seq"], :, st["t_pos"]] = x.transpose(0, 1)


def _attend_plain(st):
    c = st["case"]
    S, hq, hkv, d, P = c["seqs"], c["hq"], c["hkv"], c["d"], c["prefix"]
    g, n = hq // hkv, len(st["t_pos"])
    own_max, tok = st["k"].shape[2], c["tok_max"]
    out, lse = st["out"], st["lse"]
    qf = st["q"].float() / math.sqrt(d)
    own_pos = P + torch.arange(own_max, device="cuda")
    for h in range(hkv):
        q = qf[:, h * g:(h + 1) * g]                                       # [n][g][d]
        # own part: tokens of a sequence side by side, short ones padded
        qs = torch.zeros((S, tok, g, d), device="cuda")
        qs[st["t_seq"], st["row"]] = q
        so = torch.bmm(qs.view(S, tok * g, d), st["k"][:, h].float().transpose(1, 2).contiguous())
        so = so.view(S, tok, g, own_max)[st["t_seq"], st["row"]]           # [n][g][own_max]
        so.masked_fill_((own_pos[None, :] > st["t_pos"][:, None])[:, None, :], -math.inf)
        sp = (q.reshape(n * g, d) @ st["pk"][h].float().T).view(n, g, P)
        top = so.amax(-1)
        if P:
            top = torch.maximum(top, sp.amax(-1))
        eo, ep = torch.exp(so - top[..., None]), torch.exp(sp - top[..., None])
        den = eo.sum(-1) + ep.sum(-1)
        es = torch.zeros((S, tok, g, own_max), device="cuda")
        es[st["t_seq"], st["row"]] = eo
        o = torch.bmm(es.view(S, tok * g, own_max), st["v"][:, h].float()).view(S, tok, g, d)[st["t_seq"], st["row"]]
        o = o + (ep.view(n * g, P) @ st["pv"][h].float()).view(n, g, d)
        out[:, h * g:(h + 1) * g] = (o / den[..., None]).to(out.dtype)
        lse[:, h * g:(h + 1) * g] = top + torch.log(den)
    return {"out": out, "lse": lse}


def _rope_out(st):
    return {"q": st["q_out"], "k": st["k_out"]} if st["case"]["hq"] else {"k": st["k_out"]}


def run(state):
    st, c = state, state["case"]
    op = c["op"]
    if own:
        fcg = st["fcg"]
        if op == "rope":
            flags = fcg.FCG_ROPE_BACKWARD if c["grad"] else 0
            q = (st["q"], st["q_out"]) if c["hq"] else (None, None)
            fcg.fcg_rope_apply(st["rope"], st["pos"], *q, st["k"], st["k_out"], flags=flags)
            return _rope_out(st)
        if op == "append":
            fcg.fcg_append(st["cache"], 0, st["h_seq"], st["h_pos"], st["k"], st["v"], rope=st["rope"], q=st["q"],
                           q_out=st["q_out"], flags=fcg.FCG_REPLACE)
            return {"q": st["q_out"], "k": st["K"], "v": st["V"]}
        if op == "graft":
            for s in range(c["seqs"]):
                fcg.fcg_cache_reset(st["cache"], s)
            fcg.fcg_graft_rope(st["cache"], st["lib"], st["rope"], st["g_seq"], st["g_seg"], st["g_dst"])
            return {"k": st["K"], "v": st["V"]}
        fcg.fcg_prefix_attend(st["cache"], 0, c["seqs"], c["prefix"], st["h_seq"], st["h_pos"], st["q"], st["out"],
                              st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if op == "rope":
        sign = -1.0 if c["grad"] else 1.0
        st["q_out"].copy_(_turn(st["q"], st["pos"], c, st["w"], sign))
        st["k_out"].copy_(_turn(st["k"], st["pos"], c, st["w"], sign))
        return _rope_out(st)
    if op == "append":
        st["q_out"].copy_(_turn(st["q"], st["t_pos"], c, st["w"]))
        _place(st, _turn(st["k"], st["t_pos"], c, st["w"]), st["v"])
        return {"q": st["q_out"], "k": st["K"], "v": st["V"]}
    if op == "graft":
        k, v = (x[:, :, st["t_src"]].transpose(1, 2) for x in (st["k"], st["v"]))
        _place(st, _turn(k, st["t_delta"], c, st["w"], m=1.0), v)
        return {"k": st["K"], "v": st["V"]}
    return _attend_plain(st)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c, p = case, _Plan(case)
    es = 4 if c["dtype"] == "f32" else 2
    L, hq, hkv, d = c["layers"], c["hq"], c["hkv"], c["d"]
    row = hkv * d * es
    n = len(p.t_pos)
    if c["op"] == "rope":
        el = L * n * (hq + hkv) * d
        return {"bytes": 2.0 * el * es + 4 * n, "flops": 3.0 * L * n * (hq + hkv) * c["rot"]}
    if c["op"] == "append":
        return {"bytes": 2.0 * L * n * (hq + 2 * hkv) * d * es, "flops": 3.0 * L * n * (hq + hkv) * c["rot"]}
    if c["op"] == "graft":
        once = sum(p.lens[g] for g in set(p.seg))
        return {"bytes": 2.0 * L * row * (once + n), "flops": 3.0 * L * n * hkv * c["rot"]}
    keys = float((p.t_pos + 1).sum())
    return {"bytes": 2.0 * row * (c["prefix"] + float(p.own_len.sum())) + 2.0 * n * hq * d * es + 4.0 * n * hq,
            "flops": 4.0 * hq * d * keys}


# ------------------------------------------------------------------ the definition in 64 bits

def _encode64(x, pos, c, sign=1, m=None):
    """x [..., n, heads, d] as complex numbers turned by their angles."""
    r, f64 = c["rot"], torch.float64
    pos = torch.as_tensor(np.asarray(pos), dtype=f64, device=x.device)
    w = torch.tensor(_freqs(c), dtype=f64, device=x.device)
    ang = sign * torch.outer(pos, w)
    turn = torch.polar(torch.full_like(ang, c["m"] if m is None else m), ang)[:, None, :]
    y = x.to(f64).clone()
    if c["layout"] == "half":
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r].contiguous()) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    return y


def _memory64(c, p, k, v):
    """The cache memory that holds k, v [L][n][hkv][d] at the tokens' places, zeros elsewhere."""
    out = []
    for x in (k, v):
        x = x.to(torch.float64)
        if c["page"]:
            m = torch.zeros((c["layers"], len(p.page_key) * 16, c["hkv"], c["d"]), dtype=torch.float64, device="cuda")
            m.index_copy_(1, torch.as_tensor(p.slot, device="cuda"), x)
            m = m.unflatten(1, (-1, 16)).transpose(2, 3)
        else:
            m = torch.zeros((c["layers"], c["seqs"] * p.T, c["hkv"], c["d"]), dtype=torch.float64, device="cuda")
            m.index_copy_(1, torch.as_tensor(p.t_seq * p.T + p.t_pos, device="cuda"), x)
            m = m.unflatten(1, (c["seqs"], p.T)).transpose(2, 3)
        out.append(m)
    return out


def exact(case, seed):
    c = case
    p, t = _tensors(c, seed)
    if c["op"] == "rope":
        sign = -1 if c["grad"] else 1
        return {key: _encode64(t[key], p.t_pos, c, sign) for key in (("q", "k") if c["hq"] else ("k",))}
    if c["op"] == "append":
        k, v = _memory64(c, p, _encode64(t["k"], p.t_pos, c), t["v"])
        return {"q": _encode64(t["q"], p.t_pos, c), "k": k, "v": v}
    if c["op"] == "graft":
        src = torch.as_tensor(p.t_src, device="cuda")
        k, v = (x.index_select(2, src).transpose(1, 2) for x in (t["k"], t["v"]))
        k, v = _memory64(c, p, _encode64(k, p.t_delta, c, m=1.0), v)
        return {"k": k, "v": v}
    hq, hkv, d, P = c["hq"], c["hkv"], c["d"], c["prefix"]
    g, f64 = hq // hkv, torch.float64
    out = torch.empty((len(p.t_pos), hq, d), dtype=f64, device="cuda")
    lse = torch.empty((len(p.t_pos), hq), dtype=f64, device="cuda")
    t0 = 0
    for s in range(c["seqs"]):
        n, own_len = int(p.n[s]), int(p.own_len[s])
        seen = torch.arange(P + own_len, device="cuda")[None, :] <= torch.as_tensor(p.t_pos[t0:t0 + n, None],
                                                                                  device="cuda")
        for h in range(hkv):
            K = torch.cat([t["pk"][h], t["k"][s, h, :own_len]]).to(f64)
            V = torch.cat([t["pv"][h], t["v"][s, h, :own_len]]).to(f64)
            for j in range(h * g, (h + 1) * g):
                z = (t["q"][t0:t0 + n, j].to(f64) @ K.T) / math.sqrt(d)
                z = torch.where(seen, z, -math.inf)
                lse[t0:t0 + n, j] = torch.logsumexp(z, -1)
                out[t0:t0 + n, j] = torch.softmax(z, -1) @ V
        t0 += n
    return {"out": out, "lse": lse}
