"""What a cache takes in and what it keeps, for timing and for comparing outputs.

Four operators and how a program uses them:

``norm``     queries and keys normalised head by head and turned to their positions in one
             pass, into tensors (``fcg_norm_rope_apply``), into a cache (``fcg_append_norm``;
             a pass writes the same positions again, as a retried span does), and the
             gradient of both inputs and of the weights (``fcg_norm_rope_backward``)
``weights``  the attention weight that a call's queries put on each cached position
             (``fcg_attend_weights``), beside attention over a shared prefix
``evict``    sequences squeezed to the positions of most weight, keys turned to their new
             positions (``fcg_evict``), here into sequences of their own, so that the source
             stays
``logp``     log probabilities of given tokens with entropy and the most likely ones
             (``fcg_token_logprobs``), and the gradient of the logits
             (``fcg_token_logprobs_backward``)

Fields of a case: ``hq``, ``hkv``, ``d``, ``dtype``, ``layers``; ``layout`` (half or pairs),
``rot`` rotated dimensions, ``theta``; ``page`` (0 contiguous, 16 paged); ``seqs`` sequences
of ``tok_min`` .. ``tok_max`` tokens a call; ``far`` the largest position; ``plan`` seed of
lengths and positions.  ``norm``: ``how`` (apply, append, grad), ``heads`` a weight vector for
each head or one for all, ``offset`` added to the weights, ``fused`` q and k are slices of one
projection output.  ``weights``: ``prefix`` shared positions, ``own_min`` .. ``own_max`` own
positions up to the call's last token.  ``evict``: lengths ``len_min`` .. ``len_max``, of which
``keep_min`` .. ``keep_max`` stay, the ``first`` and the ``recent`` ones always.  ``logp``:
``n`` rows of ``vocab`` logits, ``pad`` elements between rows, ``mask`` the share of logits
that are -inf, ``top`` alternatives, ``grad`` the backward pass.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BASE = dict(hq=32, hkv=8, d=128, dtype="bf16", layers=1, layout="half", rot=128, theta=1e6, page=0, seqs=1, tok_min=1,
             tok_max=1, far=4096, plan=1, how="apply", heads=False, offset=0.0, fused=False, prefix=0, own_min=0,
             own_max=0, len_min=0, len_max=0, keep_min=0, keep_max=0, first=0, recent=0, n=0, vocab=0, pad=0, mask=0.0,
             top=0, grad=False)
_EPS = 1e-6


def _case(name, op, **more):
    return dict(_BASE, name=name, op=op, **more)


def listed():
    return [
        # the smallest call: one decode token of a model that normalises its queries and keys, into a page
        _case("norm-token", "norm", how="append", page=16, far=6000),
        # the queries and keys of a batch of prompts, slices of a fused projection
        _case("norm-prompt", "norm", fused=True, seqs=4, tok_min=900, tok_max=1300, far=8192),
        # training: the gradient of queries, keys and weights of such a batch, fp32, a weight vector for each head,
        # 96 of 128 dimensions rotated
        _case("norm-grad-f32", "norm", how="grad", hq=16, hkv=4, dtype="f32", rot=96, theta=1e4, heads=True, offset=1.0,
              seqs=4, tok_min=900, tok_max=1300, far=8192),
        # the smallest: three candidates of a small fp32 model after ~450 shared tokens
        _case("weights-tiny-f32", "weights", hq=4, hkv=2, d=64, dtype="f32", page=16, seqs=3, prefix=449, own_min=1,
              own_max=40),
        # one decode step of 64 candidate programs over one stitched context of ~4.3K tokens
        _case("weights-step", "weights", page=16, seqs=64, prefix=4321, own_min=1, own_max=300),
        # the patch prompts of 32 tasks over a shared context: 64 tokens each
        _case("weights-patch", "weights", page=16, seqs=32, prefix=6007, tok_min=64, tok_max=64, own_min=64,
              own_max=300),
        # the context of one interactive task squeezed to a quarter, all layers
        _case("evict-task", "evict", layers=32, len_min=4321, len_max=4321, keep_min=1111, keep_max=1111, first=64,
              recent=256),
        # a paged batch squeezed, half of each head rotated in neighbouring pairs
        _case("evict-batch", "evict", layers=4, page=16, seqs=16, layout="pairs", rot=64, theta=1e4, len_min=2000,
              len_max=6000, keep_min=1000, keep_max=2000, first=4, recent=128),
        # one decode token: its log probability and twenty alternatives
        _case("logp-token", "logp", n=1, vocab=131072, top=20),
        # a decode step of a batch under a grammar that rules most tokens out
        _case("logp-step", "logp", n=64, vocab=131072, pad=64, mask=0.9, top=20),
        # the perplexity of retrieved functions: every token of theirs, fp32 logits
        _case("logp-functions-f32", "logp", n=3001, vocab=50021, dtype="f32", pad=3),
        # training: the gradient of log probabilities with an entropy term
        _case("logp-grad", "logp", n=1501, vocab=100003, grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "weights", "evict", "logp"])
    c = dict(_BASE, op=op, plan=rng.randrange(1 << 20))
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (16, 4, 64), (8, 8, 64), (16, 1, 128), (4, 2, 64), (16, 8, 128)])
    c.update(hq=hq, hkv=hkv, d=d, theta=rng.choice([1e4, 1e6]))
    if rng.random() < 0.3:
        c["dtype"] = "f32"
    c["layout"] = rng.choice(["half", "pairs"])
    c["rot"] = rng.choice([d, d, d // 2, d // 4, d - 16, 16])
    c["page"] = rng.choice([0, 16])
    es = 4 if c["dtype"] == "f32" else 2
    if op == "norm":
        c["how"] = rng.choice(["apply", "append", "grad"])
        c["heads"] = rng.random() < 0.5
        c["offset"] = rng.choice([0.0, 1.0])
        c["fused"] = rng.random() < 0.5
        c["seqs"] = _log_int(rng, 1, 64)
        c["layers"] = _log_int(rng, 1, 32)
        row = (hq + 2 * hkv) * d * es * 2 * c["layers"]
        c["tok_max"] = _log_int(rng, 1, max(1, min(2000, int(1.2e8 / (row * c["seqs"])))))
        c["tok_min"] = rng.randint(1, c["tok_max"])
        c["far"] = _log_int(rng, 800, 100000)
        if c["how"] == "append":   # the cache holds the tokens and where they start
            c["far"] = min(c["far"], max(c["tok_max"] + 1, int(3e8 / (hkv * d * es * 2 * c["layers"] * c["seqs"]))))
    elif op == "weights":
        c["seqs"] = _log_int(rng, 1, 64)
        c["tok_max"] = 1 if rng.random() < 0.5 else _log_int(rng, 2, 128)
        c["tok_min"] = rng.randint(1, c["tok_max"])
        c["prefix"] = _log_int(rng, 16, 22000) if rng.random() < 0.9 else 0
        c["own_max"] = _log_int(rng, c["tok_max"], max(c["tok_max"], 1000))
        c["own_min"] = rng.randint(c["tok_max"], c["own_max"])
        lim = 1e11 if es == 2 else 1e10
        while c["seqs"] > 1 and 2.0 * hq * d * c["seqs"] * c["tok_max"] * (c["prefix"] + c["own_max"]) > lim:
            c["seqs"] = (c["seqs"] + 1) // 2
    elif op == "evict":
        c["seqs"] = _log_int(rng, 1, 16)
        c["len_max"] = _log_int(rng, 2, 20000)
        c["len_min"] = rng.randint(1, c["len_max"])
        c["keep_max"] = _log_int(rng, 1, c["len_max"])
        c["keep_min"] = rng.randint(1, c["keep_max"])
        c["first"] = rng.choice([0, 4, 64])
        c["recent"] = rng.choice([0, 32, 256])
        c["layers"] = max(1, min(_log_int(rng, 1, 32), int(1.5e9 / (c["seqs"] * c["len_max"] * hkv * d * es * 2))))
        while c["seqs"] > 1 and c["seqs"] * c["len_max"] * hkv * d * es * 2 * c["layers"] > 1.6e9:
            c["seqs"] = (c["seqs"] + 1) // 2
    else:
        c["vocab"] = _log_int(rng, 1000, 152000)
        c["n"] = _log_int(rng, 1, min(4096, int((1.5e8 if es == 4 else 3e8) / c["vocab"])))
        c["pad"] = rng.choice([0, 0, 1, 64])
        c["mask"] = rng.choice([0.0, 0.0, 0.5, 0.99])
        c["grad"] = rng.random() < 0.4
        c["top"] = 0 if c["grad"] else rng.choice([0, 1, 5, 20, 64])
        if c["grad"]:
            c["n"] = max(1, c["n"] // 2)
    return c


# ------------------------------------------------------------------ sizes and positions (from the case alone)

def _freqs(c):
    return [c["theta"] ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]


class _Plan:
    def __init__(self, c):
        rng = np.random.default_rng(c["plan"])
        S = c["seqs"]
        if c["op"] == "logp":
            return
        if c["op"] == "evict":
            self.len = rng.integers(c["len_min"], c["len_max"], size=S, endpoint=True).astype(np.int64)
            self.keep = np.minimum(self.len, rng.integers(c["keep_min"], c["keep_max"], size=S, endpoint=True)).astype(np.int64)
            self.T = -(-int(self.len.max()) // 16) * 16
            self.J = int(self.keep.max())
            pages = -(-self.len // 16)
            self.page0 = np.concatenate([[0], np.cumsum(pages)]).astype(np.int64)       # first page of a source
            self.n_src = int(pages.sum())
            dpages = -(-self.keep // 16)
            self.dpage0 = self.n_src + np.concatenate([[0], np.cumsum(dpages)]).astype(np.int64)
            self.n_pages = self.n_src + int(dpages.sum())
            self.t_seq = np.repeat(np.arange(S), self.keep)                             # kept rows: sequence, place
            self.t_to = np.concatenate([np.arange(k) for k in self.keep]).astype(np.int64)
            return
        n = rng.integers(c["tok_min"], c["tok_max"], size=S, endpoint=True)
        if c["op"] == "weights":
            self.own_len = np.maximum(n, rng.integers(c["own_min"], c["own_max"], size=S, endpoint=True)).astype(np.int64)
            start = c["prefix"] + self.own_len - n
            self.T = max(16, -(-(c["prefix"] + int(self.own_len.max())) // 16) * 16)
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

    def __call__(self, *shape, scale=1.0, at=0.0):
        return (torch.randn(shape, generator=self.g, device="cuda") * scale + at).to(self.dt)

    def f32(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def below(self, top, *shape):
        return torch.randint(top, shape, generator=self.g, device="cuda", dtype=torch.int32)


def _tensors(c, seed):
    """The values of a case, drawn in a fixed order."""
    p, vals = _Plan(c), _Values(c, seed)
    L, S, d, hq, hkv = c["layers"], c["seqs"], c["d"], c["hq"], c["hkv"]
    t = {}
    if c["op"] == "norm":
        n = len(p.t_pos)
        if c["fused"]:      # slices of one projection output [L][n][hq + 2 hkv][d]
            x = vals(L, n, hq + 2 * hkv, d, scale=2.0)
            t["q"], t["k"], t["v"] = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        else:
            t["q"], t["k"], t["v"] = vals(L, n, hq, d, scale=2.0), vals(L, n, hkv, d, scale=2.0), vals(L, n, hkv, d)
        for key, heads in (("qw", hq), ("kw", hkv)):
            t[key] = vals(L, heads if c["heads"] else 1, d, scale=0.1, at=1.0 - c["offset"])
        if c["how"] == "grad":
            t["gq"], t["gk"] = vals(L, n, hq, d), vals(L, n, hkv, d)
    elif c["op"] == "weights":
        own_max = int(p.own_len.max())
        t["q"] = vals(len(p.t_pos), hq, d)
        t["pk"], t["k"] = vals(hkv, c["prefix"], d), vals(S, hkv, own_max, d)
        t["held"] = 1e-4 * vals.uniform(S + 1, hkv, p.T)     # what the rows hold where nothing attends
    elif c["op"] == "evict":
        shape = (L, p.n_pages, hkv, 16, d) if c["page"] else (L, 2 * S, hkv, p.T, d)
        t["K"], t["V"] = vals(*shape), vals(*shape)
        # accumulated weights: a few large, many small, some positions that nothing attended to
        w = torch.exp(2.0 * vals.f32(L, 2 * S, hkv, p.T))
        t["w"] = torch.where(vals.uniform(L, 2 * S, hkv, p.T) < 0.2, torch.zeros_like(w), w)
    else:
        n, V = c["n"], c["vocab"]
        x = vals(n, V + c["pad"], scale=2.5)
        if c["mask"]:
            x = torch.where(vals.uniform(n, V + c["pad"]) < c["mask"], torch.full_like(x, -math.inf), x)
            x[:, V // 2] = 1.5      # something is always allowed
        t["x"] = x[:, :V]
        t["target"] = vals.below(V, n)
        if c["mask"]:
            t["target"].fill_(V // 2)
        if c["grad"]:
            t["g_logprob"], t["g_entropy"], t["g_lse"] = (vals.f32(n) for _ in range(3))
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


def _row_stats(x):
    """lse and entropy of rows, as the forward pass of a training step leaves them (64 bits, rounded once)."""
    x = x.to(torch.float64)
    lse = torch.logsumexp(x, -1)
    lp = x - lse[:, None]
    ent = -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(-1)
    return lse.float(), ent.float()


def _lse_of(c, p, t):
    """The log-sum-exp that attention over the same keys returns [n][hq]."""
    hq, hkv, d, P = c["hq"], c["hkv"], c["d"], c["prefix"]
    g, n = hq // hkv, len(p.t_pos)
    out = torch.empty((n, hkv, g), device="cuda")
    t0 = 0
    for s in range(c["seqs"]):
        m, own_len = int(p.n[s]), int(p.own_len[s])
        keys = torch.cat([t["pk"], t["k"][s, :, :own_len]], dim=1).float()
        q = t["q"][t0:t0 + m].float().view(m, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, m * g, d)
        z = torch.bmm(q, keys.transpose(1, 2).contiguous()).view(hkv, m, g, P + own_len) / math.sqrt(d)
        late = torch.arange(P + own_len, device="cuda")[None, :] > torch.as_tensor(p.t_pos[t0:t0 + m, None], device="cuda")
        z.masked_fill_(late[None, :, None, :], -math.inf)
        out[t0:t0 + m] = torch.logsumexp(z, -1).permute(1, 0, 2)
        t0 += m
    return out.view(n, hq)


def prepare(case, seed):
    c = case
    p, t = _tensors(c, seed)
    dt = _DT[c["dtype"]]
    dev = "cuda"
    L, S, hq, hkv, d = c["layers"], c["seqs"], c["hq"], c["hkv"], c["d"]
    st = {"case": c, "plan": p, **t}
    paged = c["page"] != 0
    if c["op"] == "logp":
        n, V = c["n"], c["vocab"]
        if c["grad"]:
            st["lse"], st["entropy"] = _row_stats(t["x"])
            st["dx"] = torch.empty((n, V), dtype=dt, device=dev)
        else:
            st["logprob"], st["entropy"], st["lse"] = (torch.empty(n, device=dev) for _ in range(3))
            st["top_id"] = torch.empty((n, c["top"]), dtype=torch.int32, device=dev)
            st["top_logprob"] = torch.empty((n, c["top"]), device=dev)
        if own:
            from paper_2606_13097_amd import fcg
            st["fcg"] = fcg
            if not c["grad"]:
                st["ws"] = torch.empty(fcg.fcg_token_logprobs_workspace(n, V, c["top"]), dtype=torch.uint8, device=dev)
        else:
            st["target"] = t["target"].long()
        return st
    if c["op"] == "norm":
        n = len(p.t_pos)
        n_pages = len(p.page_key)
        shape = (L, n_pages, hkv, 16, d) if paged else (L, S, hkv, p.T, d)
        if c["how"] == "grad":
            st["dq"], st["dk"] = torch.empty((L, n, hq, d), dtype=dt, device=dev), torch.empty((L, n, hkv, d), dtype=dt, device=dev)
            st["dqw"], st["dkw"] = (torch.empty(t[key].shape, device=dev) for key in ("qw", "kw"))
        else:
            st["q_out"] = torch.empty((L, n, hq, d), dtype=dt, device=dev)
        if c["how"] == "apply":
            st["k_out"] = torch.empty((L, n, hkv, d), dtype=dt, device=dev)
        if c["how"] != "append":
            st["pos"] = torch.as_tensor(p.t_pos, dtype=torch.int32, device=dev)
    if c["op"] == "weights":
        st["lse"] = _lse_of(c, p, t)
    if c["op"] == "evict":
        n_pages = p.n_pages
        shape = t["K"].shape
        st["kept"] = torch.full((L, S, hkv, p.J), -1, dtype=torch.int32, device=dev)
        # the squeezed sequences hold nothing yet
        st["new"] = slice(p.n_src, p.n_pages) if paged else slice(S, 2 * S)
        for m in (t["K"], t["V"]):
            m[:, st["new"]] = 0
    if not own:
        st["w_freq"] = torch.tensor(_freqs(c), dtype=torch.float64, device=dev)
        for key in ("t_seq", "t_pos", "t_to", "slot", "page0", "dpage0", "len", "keep", "own_len"):
            if hasattr(p, key):
                st[key] = torch.as_tensor(getattr(p, key), device=dev)
        if c["op"] == "norm" and c["how"] == "append":
            st["K"], st["V"] = (torch.zeros(shape, dtype=dt, device=dev) for _ in range(2))
        if c["op"] == "weights":     # row of each token in a [S][tok_max] arrangement
            st["row"] = torch.as_tensor(np.concatenate([np.arange(k) for k in p.n]), device=dev)
        return st
    from paper_2606_13097_amd import fcg
    st["fcg"] = fcg
    desc = fcg.model_desc(L, max(hq, hkv), hkv, d, c["theta"], c["dtype"])
    layout = fcg.FCG_ROPE_HALF if c["layout"] == "half" else fcg.FCG_ROPE_PAIRS
    if c["op"] != "weights":
        st["rope"] = fcg.fcg_rope_create(c["rot"], c["theta"], layout=layout)
    if c["op"] == "norm":
        st["q_norm"], st["k_norm"] = (fcg.Norm(t[key], eps=_EPS, offset=c["offset"]) for key in ("qw", "kw"))
        if c["how"] == "append":
            st["cache"] = fcg.fcg_cache_create(desc, S, p.T, c["page"], n_pages if paged else 0)
            st["K"], st["V"] = _cache_memory(fcg, st["cache"], shape, dt, st["cache"])
            st["K"].zero_(), st["V"].zero_()
            st["h_seq"], st["h_pos"] = p.t_seq.astype(np.int32), p.t_pos.astype(np.int32)
        if c["how"] == "grad":
            st["ws"] = torch.empty(fcg.fcg_norm_rope_workspace(L, len(p.t_pos), hq, hkv, d), dtype=torch.uint8, device=dev)
        return st
    if c["op"] == "weights":
        # the cache as a program leaves it: the prefix in sequence S, each task's own tokens after it
        sq = np.concatenate([np.full(c["prefix"], S)] + [np.full(n, s) for s, n in enumerate(p.own_len)])
        ps = np.concatenate([np.arange(c["prefix"])] + [np.arange(c["prefix"], c["prefix"] + n) for n in p.own_len])
        total = sum(-(-(c["prefix"] + n) // 16) for n in p.own_len) + -(-max(c["prefix"], 1) // 16)
        st["cache"] = cache = fcg.fcg_cache_create(desc, S + 1, p.T, c["page"], total if paged else 0)
        fcg.fcg_append(cache, 0, sq, ps)
        shape = (1, total, hkv, 16, d) if paged else (1, S + 1, hkv, p.T, d)
        mem = _cache_memory(fcg, cache, shape, dt, cache)[0]
        for s in range(S + 1):
            x, at = (t["pk"], 0) if s == S else (t["k"][s, :, :int(p.own_len[s])], c["prefix"])
            if not x.shape[1]:
                continue
            if paged:
                pt, _, _ = fcg.fcg_cache_export_layout(cache, s, 0)
                pos = np.arange(at, at + x.shape[1])
                page = torch.as_tensor(pt[pos // 16].astype(np.int64), device=dev)
                mem[0][page, :, torch.as_tensor(pos % 16, device=dev)] = x.transpose(0, 1)
            else:
                mem[0, s, :, at:at + x.shape[1]] = x
        st["h_seq"], st["h_pos"] = p.t_seq.astype(np.int32), p.t_pos.astype(np.int32)
        st.update(pk=None, k=None)
        return st
    # evict: sources 0 .. S - 1 written from position 0, sequences S .. 2 S - 1 empty
    st["cache"] = cache = fcg.fcg_cache_create(desc, 2 * S, p.T, c["page"], n_pages if paged else 0)
    sq = np.repeat(np.arange(S), p.len)
    fcg.fcg_append(cache, 0, sq, np.concatenate([np.arange(n) for n in p.len]), n_layers=L)
    for mem, key in zip(_cache_memory(fcg, cache, shape, dt, cache), ("K", "V")):
        mem.copy_(t[key])
        st[key] = mem
    st["h_src"], st["h_dst"] = np.arange(S, dtype=np.int32), np.arange(S, 2 * S, dtype=np.int32)
    st["h_keep"] = p.keep.astype(np.int32)
    return st


# ------------------------------------------------------------------ one pass

def _cos_sin(at, w):
    """cos and sin of the angles of positions (or distances) `at`, taken in 64 bits."""
    a = at.to(torch.float64)[..., None] * w
    return a.cos().float(), a.sin().float()


def _turn(x, cos, sin, c):
    """The rotary turn of x [..., d] in 32 bits; cos, sin [..., rot / 2]."""
    r = c["rot"]
    if c["layout"] == "half":
        xa, xb = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([xa * cos - xb * sin, xb * cos + xa * sin, x[..., r:]], dim=-1)
    xa, xb = x[..., 0:r:2], x[..., 1:r:2]
    y = torch.stack([xa * cos - xb * sin, xb * cos + xa * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _norm_plain(x, w, c, cos, sin):
    """x [L][n][heads][d], w [L][heads or 1][d]."""
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + _EPS)
    return _turn(x32 * r * (w.float() + c["offset"])[:, None], cos, sin, c).to(x.dtype)


def _norm_grad_plain(x, w, gy, c, cos, sin):
    x32 = x.float()
    r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + _EPS)
    xn = x32 * r
    gn = _turn(gy.float(), cos, -sin, c)                       # gradient before the turn
    gw = (gn * xn).sum(1)                                      # [L][heads][d]
    if not c["heads"]:
        gw = gw.sum(1, keepdim=True)
    gx = gn * (w.float() + c["offset"])[:, None]
    dx = r * (gx - xn * (gx * xn).mean(-1, keepdim=True))
    return dx.to(x.dtype), gw


def _place(st, k, v):
    """k, v [L][n][hkv][d] into the cache memory at the tokens' places."""
    for mem, x in ((st["K"], k), (st["V"], v)):
        if st["case"]["page"]:
            mem[:, st["slot"] // 16, :, st["slot"] % 16] = x.transpose(0, 1)
        else:
            mem[:, st["t_seq"], :, st["t_pos"]] = x.transpose(0, 1)


def _weights_plain(st):
    c = st["case"]
    S, hq, hkv, d, P = c["seqs"], c["hq"], c["hkv"], c["d"], c["prefix"]
    g, n = hq // hkv, len(st["t_pos"])
    own_max, tok = st["k"].shape[2], c["tok_max"]
    held = st["held"]
    q = (st["q"].float() / math.sqrt(d)).view(n, hkv, g, d)
    lse = st["lse"].view(n, hkv, g)
    if P:
        z = torch.bmm(q.permute(1, 0, 2, 3).reshape(hkv, n * g, d), st["pk"].float().transpose(1, 2).contiguous())
        z -= lse.permute(1, 0, 2).reshape(hkv, n * g, 1)
        held[S, :, :P] = z.exp_().sum(1)
    # own part: tokens of a sequence side by side, short ones padded
    qs = torch.zeros((S, tok, hkv, g, d), device="cuda")
    ls = torch.zeros((S, tok, hkv, g), device="cuda")
    last = torch.full((S, tok), -1, dtype=torch.int64, device="cuda")     # the last own key that a row sees
    qs[st["t_seq"], st["row"]], ls[st["t_seq"], st["row"]] = q, lse
    last[st["t_seq"], st["row"]] = st["t_pos"] - P
    z = torch.bmm(qs.permute(0, 2, 1, 3, 4).reshape(S * hkv, tok * g, d),
                  st["k"].float().transpose(2, 3).contiguous().view(S * hkv, d, own_max)).view(S, hkv, tok, g, own_max)
    j = torch.arange(own_max, device="cuda")
    z = torch.exp(z - ls.permute(0, 2, 1, 3)[..., None])
    z = torch.where((j <= last[:, :, None])[:, None, :, None, :], z, 0.0).sum((2, 3))       # [S][hkv][own_max]
    mine = (j < st["own_len"][:, None])[:, None, :]
    held[:S, :, P:P + own_max] = torch.where(mine, z, held[:S, :, P:P + own_max])
    return {"weights": held}


def _evict_plain(st):
    c = st["case"]
    L, S, hkv = c["layers"], c["seqs"], c["hkv"]
    n, keep = st["len"][:, None], st["keep"][:, None]
    T, J = st["w"].shape[3], st["kept"].shape[3]
    pos = torch.arange(T, device="cuda")
    first = torch.minimum(keep, torch.full_like(keep, c["first"]))
    recent = torch.minimum(keep - first, torch.full_like(keep, c["recent"]))
    always = (pos < first) | ((pos >= n - recent) & (pos < n))                              # [S][T]
    score = st["w"][:, :S].masked_fill(always[:, None], math.inf).masked_fill((pos >= n)[:, None], -math.inf)
    order = torch.sort(score, dim=3, descending=True, stable=True).indices                  # ties: lowest first
    out = torch.arange(T, device="cuda") >= keep                                            # [S][T] ranks that go
    kept = torch.sort(order.masked_fill(out[:, None], T), dim=3).values[..., :J]            # [L][S][hkv][J]
    st["kept"].copy_(torch.where(kept < T, kept, -1))
    ts, to = st["t_seq"], st["t_to"]
    at = kept.transpose(1, 2)[:, :, ts, to]                                                 # [L][hkv][rows]
    l = torch.arange(L, device="cuda")[:, None, None]
    h = torch.arange(hkv, device="cuda")[None, :, None]
    if c["page"]:
        src = (l, st["page0"][ts] + at // 16, h, at % 16)
        dst = (l, st["dpage0"][ts] + to // 16, h, to % 16)
    else:
        src, dst = (l, ts, h, at), (l, S + ts, h, to)
    cos, sin = _cos_sin(to - at, st["w_freq"])
    st["K"][dst] = _turn(st["K"][src].float(), cos, sin, c).to(st["K"].dtype)
    st["V"][dst] = st["V"][src]
    st["w"][:, S:] = 0
    st["w"][l, S + ts, h, to] = st["w"][l, ts, h, at]
    return _evict_out(st)


def _evict_out(st):
    S = st["case"]["seqs"]
    return {"kept": st["kept"], "k": st["K"][:, st["new"]], "v": st["V"][:, st["new"]], "weights": st["w"][:, S:]}


def _logp_plain(st):
    c = st["case"]
    x = st["x"].float()
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    st["lse"].copy_(lse[:, 0])
    st["logprob"].copy_((x.gather(1, st["target"][:, None]) - lse)[:, 0])
    below = torch.where(e > 0, x - top, 0.0)
    st["entropy"].copy_((torch.log(total) - (e * below).sum(-1, keepdim=True) / total)[:, 0])
    if c["top"]:
        # one whole number for each logit: order of its value, then of its index from behind
        bits = (x + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) + ((1 << 20) - 1
                                                                             - torch.arange(x.shape[1], device="cuda"))
        ids = (1 << 20) - 1 - (torch.topk(key, c["top"], dim=1).values & ((1 << 20) - 1))
        st["top_id"].copy_(ids)
        st["top_logprob"].copy_(x.gather(1, ids) - lse)
    return _logp_out(st)


def _logp_grad_plain(st):
    x = st["x"].float()
    lp = x - st["lse"][:, None]
    p = lp.exp()
    gl, gh, gs = (st[key][:, None] for key in ("g_logprob", "g_entropy", "g_lse"))
    dx = torch.where(p > 0, p * (gs - gl - gh * (lp + st["entropy"][:, None])), 0.0)
    dx.scatter_add_(1, st["target"][:, None], gl)
    st["dx"].copy_(dx)
    return {"dx": st["dx"]}


def _logp_out(st):
    return {key: st[key] for key in ("logprob", "entropy", "lse", "top_id", "top_logprob")[:5 if st["case"]["top"] else 3]}


def _norm_out(st):
    c = st["case"]
    if c["how"] == "apply":
        return {"q": st["q_out"], "k": st["k_out"]}
    if c["how"] == "append":
        return {"q": st["q_out"], "k": st["K"], "v": st["V"]}
    return {"q": st["dq"], "k": st["dk"], "qw": st["dqw"], "kw": st["dkw"]}


def run(state):
    st, c = state, state["case"]
    op = c["op"]
    if own:
        fcg = st["fcg"]
        if op == "norm":
            if c["how"] == "apply":
                fcg.fcg_norm_rope_apply(st["rope"], st["pos"], st["q"], st["q_norm"], st["q_out"], st["k"], st["k_norm"],
                                        st["k_out"])
            elif c["how"] == "append":
                fcg.fcg_append_norm(st["cache"], 0, st["h_seq"], st["h_pos"], st["k"], st["v"], st["k_norm"],
                                    rope=st["rope"], q=st["q"], q_norm=st["q_norm"], q_out=st["q_out"],
                                    flags=fcg.FCG_REPLACE)
            else:
                fcg.fcg_norm_rope_backward(st["rope"], st["pos"], st["q"], st["q_norm"], st["gq"], st["dq"], st["dqw"],
                                           st["k"], st["k_norm"], st["gk"], st["dk"], st["dkw"], workspace=st["ws"])
            return _norm_out(st)
        if op == "weights":
            fcg.fcg_attend_weights(st["cache"], 0, c["seqs"], c["prefix"], st["h_seq"], st["h_pos"], st["q"], st["lse"],
                                   st["held"])
            return {"weights": st["held"]}
        if op == "evict":
            fcg.fcg_evict(st["cache"], st["h_src"], st["h_dst"], st["h_keep"], st["w"], first=c["first"],
                          recent=c["recent"], rope=st["rope"], kept=st["kept"])
            return _evict_out(st)
        if c["grad"]:
            fcg.fcg_token_logprobs_backward(st["x"], st["target"], st["lse"], st["entropy"], st["dx"],
                                            g_logprob=st["g_logprob"], g_entropy=st["g_entropy"], g_lse=st["g_lse"])
            return {"dx": st["dx"]}
        top = (st["top_id"], st["top_logprob"]) if c["top"] else (None, None)
        fcg.fcg_token_logprobs(st["x"], st["target"], st["logprob"], st["entropy"], st["lse"], *top, workspace=st["ws"])
        return _logp_out(st)
    if op == "norm":
        pos = st["t_pos"] if c["how"] == "append" else st["pos"]
        cos, sin = _cos_sin(pos[:, None], st["w_freq"])          # [n][1][rot / 2]
        if c["how"] == "grad":
            for x, w, gy, dx, dw in (("q", "qw", "gq", "dq", "dqw"), ("k", "kw", "gk", "dk", "dkw")):
                a, b = _norm_grad_plain(st[x], st[w], st[gy], c, cos, sin)
                st[dx].copy_(a), st[dw].copy_(b)
            return _norm_out(st)
        st["q_out"].copy_(_norm_plain(st["q"], st["qw"], c, cos, sin))
        k = _norm_plain(st["k"], st["kw"], c, cos, sin)
        if c["how"] == "apply":
            st["k_out"].copy_(k)
        else:
            _place(st, k, st["v"])
        return _norm_out(st)
    if op == "weights":
        return _weights_plain(st)
    if op == "evict":
        return _evict_plain(st)
    return _logp_grad_plain(st) if c["grad"] else _logp_plain(st)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c, p = case, _Plan(case)
    es = 4 if c["dtype"] == "f32" else 2
    L, S, hq, hkv, d = c["layers"], c["seqs"], c["hq"], c["hkv"], c["d"]
    if c["op"] == "norm":
        n = len(p.t_pos)
        w = L * d * (hq + hkv if c["heads"] else 2)
        el = L * n * (hq + hkv) * d
        if c["how"] == "grad":
            return {"bytes": 3.0 * el * es + w * (es + 4.0) + 4 * n, "flops": 10.0 * el + 3.0 * L * n * (hq + hkv) * c["rot"]}
        moved = el + (L * n * hkv * d if c["how"] == "append" else 0)
        return {"bytes": 2.0 * moved * es + w * es + 4 * n, "flops": 4.0 * el + 3.0 * L * n * (hq + hkv) * c["rot"]}
    if c["op"] == "weights":
        n, keys = len(p.t_pos), c["prefix"] + float(p.own_len.sum())
        return {"bytes": hkv * d * es * keys + n * hq * (d * es + 4.0) + 4.0 * hkv * keys,
                "flops": 2.0 * hq * d * float((p.t_pos + 1).sum())}
    if c["op"] == "evict":
        rows = L * hkv * float(p.keep.sum())
        return {"bytes": rows * (4.0 * d * es + 8.0) + 4.0 * L * hkv * (float(p.len.sum()) + S * p.T),
                "flops": 3.0 * rows * c["rot"]}
    el = float(c["n"]) * c["vocab"]
    return {"bytes": el * es * (2.0 if c["grad"] else 1.0) + c["n"] * (16.0 + 8.0 * c["top"]), "flops": 5.0 * el}


# ------------------------------------------------------------------ the definition in 64 bits

def _turn64(x, ang, c):
    """x [..., d] as complex numbers turned by ang [..., rot / 2]."""
    r = c["rot"]
    turn = torch.polar(torch.ones_like(ang), ang)
    y = x.clone()
    if c["layout"] == "half":
        z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_norm(c, p, t):
    f64 = torch.float64
    w = torch.tensor(_freqs(c), dtype=f64, device="cuda")
    ang = torch.outer(torch.as_tensor(p.t_pos, dtype=f64, device="cuda"), w)[:, None, :]

    def forward(x, weight):
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["d"] + _EPS)
        return _turn64(x * (weight + c["offset"]).unsqueeze(1), ang, c)

    if c["how"] != "grad":
        q, k = forward(t["q"].to(f64), t["qw"].to(f64)), forward(t["k"].to(f64), t["kw"].to(f64))
        if c["how"] == "apply":
            return {"q": q, "k": k}
        out = []
        for x in (k, t["v"].to(f64)):
            if c["page"]:
                m = torch.zeros((c["layers"], len(p.page_key) * 16, c["hkv"], c["d"]), dtype=f64, device="cuda")
                m.index_copy_(1, torch.as_tensor(p.slot, device="cuda"), x)
                out.append(m.unflatten(1, (-1, 16)).transpose(2, 3))
            else:
                m = torch.zeros((c["layers"], c["seqs"] * p.T, c["hkv"], c["d"]), dtype=f64, device="cuda")
                m.index_copy_(1, torch.as_tensor(p.t_seq * p.T + p.t_pos, device="cuda"), x)
                out.append(m.unflatten(1, (c["seqs"], p.T)).transpose(2, 3))
        return {"q": q, "k": out[0], "v": out[1]}
    res = {}
    for x, wt, gy in (("q", "qw", "gq"), ("k", "kw", "gk")):     # the derivative that autograd takes of the definition
        a, b = t[x].to(f64).requires_grad_(), t[wt].to(f64).requires_grad_()
        with torch.enable_grad():
            n = a / torch.sqrt(a.square().sum(-1, keepdim=True) / c["d"] + _EPS) * (b + c["offset"]).unsqueeze(1)
        back = _turn64(t[gy].to(f64), -ang, c)                   # a rotation's transpose is its inverse
        res[x], res[wt] = torch.autograd.grad(n, (a, b), back)
    return res


def _exact_weights(c, p, t):
    hq, hkv, d, P, S = c["hq"], c["hkv"], c["d"], c["prefix"], c["seqs"]
    g, f64 = hq // hkv, torch.float64
    out = t["held"].to(f64).clone()
    out[S, :, :P] = 0.0
    lse = _lse_of(c, p, t).to(f64)
    t0 = 0
    for s in range(S):
        n, own_len = int(p.n[s]), int(p.own_len[s])
        seen = torch.arange(P + own_len, device="cuda")[None, :] <= torch.as_tensor(p.t_pos[t0:t0 + n, None], device="cuda")
        out[s, :, P:P + own_len] = 0.0
        for h in range(hkv):
            K = torch.cat([t["pk"][h], t["k"][s, h, :own_len]]).to(f64)
            for i in range(h * g, (h + 1) * g):
                z = (t["q"][t0:t0 + n, i].to(f64) @ K.T) / math.sqrt(d) - lse[t0:t0 + n, i, None]
                w = torch.where(seen, z.exp(), 0.0).sum(0)
                out[S, h, :P] += w[:P]
                out[s, h, P:P + own_len] += w[P:]
        t0 += n
    return {"weights": out}


def _exact_evict(c, p, t):
    L, S, hkv, f64 = c["layers"], c["seqs"], c["hkv"], torch.float64
    new = slice(p.n_src, p.n_pages) if c["page"] else slice(S, 2 * S)
    K, V = (torch.zeros_like(t[key][:, new], dtype=f64) for key in ("K", "V"))
    W = torch.zeros((L, S, hkv, p.T), dtype=f64, device="cuda")
    freq = torch.tensor(_freqs(c), dtype=f64, device="cuda")
    w = t["w"].cpu().numpy()
    for s in range(S):
        n, keep = int(p.len[s]), int(p.keep[s])
        first = min(keep, c["first"])
        recent = min(keep - first, c["recent"])
        mid = w[:, s, :, first:n - recent].reshape(L * hkv, -1)
        order = np.lexsort((np.broadcast_to(np.arange(mid.shape[1]), mid.shape), -mid), axis=1)
        chosen = first + np.sort(order[:, :keep - first - recent], axis=1)
        ends = [np.broadcast_to(np.arange(a, b), (L * hkv, b - a)) for a, b in ((0, first), (n - recent, n))]
        at = torch.as_tensor(np.concatenate([ends[0], chosen, ends[1]], axis=1).reshape(L, hkv, keep), device="cuda")
        to = torch.arange(keep, device="cuda")
        if c["page"]:
            page, d = int(p.page0[s]), c["d"]
            span = slice(page, page + -(-n // 16))
            k, v = (t[key][:, span].transpose(1, 2).reshape(L, hkv, -1, d) for key in ("K", "V"))
        else:
            k, v = t["K"][:, s], t["V"][:, s]
        pick = at[..., None].expand(-1, -1, -1, c["d"])
        k, v = k.gather(2, pick).to(f64), v.gather(2, pick).to(f64)
        k = _turn64(k, (to - at).to(f64)[..., None] * freq, c)
        W[:, s, :, :keep] = torch.as_tensor(w[:, s], device="cuda").gather(2, at).to(f64)
        for mem, x in ((K, k), (V, v)):
            if c["page"]:
                x = torch.nn.functional.pad(x, (0, 0, 0, -keep % 16)).unflatten(2, (-1, 16)).transpose(1, 2)
                at0 = int(p.dpage0[s]) - p.n_src
                mem[:, at0:at0 + x.shape[1]] = x
            else:
                mem[:, s, :, :keep] = x
    return {"kept": None, "k": K, "v": V, "weights": W}


def _exact_logp(c, p, t):
    x = t["x"].to(torch.float64)
    at = t["target"].long()[:, None]
    if c["grad"]:
        lse, ent = (v.to(torch.float64)[:, None] for v in _row_stats(t["x"]))
        gl, gh, gs = (t[key].to(torch.float64)[:, None] for key in ("g_logprob", "g_entropy", "g_lse"))
        p = torch.exp(x - lse)
        dx = p * (gs - gl) - gh * (torch.special.xlogy(p, p) + p * ent)
        return {"dx": dx.scatter_add(1, at, gl)}
    lse = torch.logsumexp(x, -1)
    prob = torch.softmax(x, -1)
    out = {"logprob": x.gather(1, at)[:, 0] - lse, "entropy": -torch.special.xlogy(prob, prob).sum(-1), "lse": lse}
    if c["top"]:
        out["top_id"] = None
        out["top_logprob"] = torch.topk(x, c["top"], dim=1).values - lse[:, None]
    return out


def exact(case, seed):
    c = case
    p, t = _tensors(c, seed)
    if c["op"] == "norm":
        return _exact_norm(c, p, t)
    if c["op"] == "weights":
        return _exact_weights(c, p, t)
    return _exact_evict(c, p, t) if c["op"] == "evict" else _exact_logp(c, p, t)
