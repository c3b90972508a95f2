"""Plain 64-bit forms of attention weight per position and of eviction by it."""
import math

import numpy as np
import torch

from paper_2606_13097_amd import fcg


def place(cache, seq, positions):
    """Index of the rows of positions of a sequence in a layer of a cache's memory tensor ([...][hkv][d] results)."""
    positions = torch.as_tensor(np.asarray(positions, dtype=np.int64))
    if not cache.page_size:
        return (seq, slice(None), positions)
    pt, _, _ = fcg.fcg_cache_export_layout(cache, seq, 0)
    return (torch.as_tensor(pt.astype(np.int64))[positions // 16], slice(None), positions % 16)


def fill_sequence(cache, mem, layer, seq, at, x):
    """Reserve positions at .. of a sequence in every layer and put rows x [n][hkv][d] there."""
    n = x.shape[0]
    if not n:
        return
    pos = np.arange(at, at + n)
    fcg.fcg_append(cache, 0, np.full(n, seq), pos, n_layers=cache.desc.n_layers)
    if cache.page_size:
        mem[layer][place(cache, seq, pos)] = x
    else:
        mem[layer, seq, :, at:at + n] = x.transpose(0, 1)


def weights64(q, keys, pre, P, seq, pos, T, hkv):
    """q [n][hq][d]; keys[s] [len][hkv][d]: the prefix (s = pre), or own keys from position P on.
    -> sums [n_seqs][hkv][T], lse [n][hq], the most rows of a sum, the largest sum |q k| / sqrt(d), where summed."""
    n, hq, d = q.shape
    g = hq // hkv
    out = torch.zeros((len(keys), hkv, T), dtype=torch.float64, device=q.device)
    attended = torch.zeros((len(keys), hkv, T), dtype=torch.bool, device=q.device)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device)
    reach = 0.0
    for t in range(n):
        s, own = int(seq[t]), int(pos[t]) - P + 1
        K = torch.cat([keys[pre][:P], keys[s][:own]]).double()
        if not len(K):
            continue
        for h in range(hkv):
            qt = q[t, h * g:(h + 1) * g].double()
            z = qt @ K[:, h].T / math.sqrt(d)
            lse[t, h * g:(h + 1) * g] = torch.logsumexp(z, -1)
            w = torch.softmax(z, -1).sum(0)
            out[pre, h, :P] += w[:P]
            out[s, h, P:P + own] += w[P:]
            reach = max(reach, float((qt.abs() @ K[:, h].abs().T).max()) / math.sqrt(d))
        attended[pre, :, :P] = True
        attended[s, :, P:P + own] = True
    return out, lse, n * g, reach, attended


def kept64(w, n, keep, first, recent):
    """Positions that stay of the n first of a weight row w (numpy float32), ascending."""
    keep = min(keep, n)
    if keep == n:
        return np.arange(n)
    f = min(keep, first)
    r = min(keep - f, recent)
    x = w[f:n - r].astype(np.float64)
    order = sorted(range(len(x)), key=lambda i: (math.isnan(x[i]), -x[i] if not math.isnan(x[i]) else 0.0, i))
    mid = sorted(f + i for i in order[:keep - f - r])
    return np.concatenate([np.arange(f), mid, np.arange(n - r, n)]).astype(np.int64)
