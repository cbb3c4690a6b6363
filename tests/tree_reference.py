"""Plain 64-bit forms of the chunk operators with sinks and trees, and of sampling; how far a kernel may be from the former by
its roundings (the terms are those of extend_reference)."""
import math

import torch

from tests.extend_reference import EPS, e4m3


def random_trees(n_new, seed, depth=8, roots=1):
    """Parents and depths of every sequence's nodes, in an order that has parents before children."""
    g = torch.Generator().manual_seed(seed)
    parents, depths = [], []
    for n in n_new:
        p, dep = [], []
        for i in range(n):
            up = -1
            if i >= roots:
                up = int(torch.randint(max(0, i - 12), i, (1,), generator=g))
                while up >= 0 and dep[up] + 1 >= depth:
                    up = p[up]
            p.append(up)
            dep.append(dep[up] + 1 if up >= 0 else 0)
        parents.append(p)
        depths.append(dep)
    return parents, depths


def ancestors(parents):
    """[t, t]: node i sees node j of its tree."""
    t = len(parents)
    m = torch.zeros((t, t), dtype=torch.bool)
    for i in range(t):
        j = i
        while j >= 0:
            m[i, j] = True
            j = parents[j]
    return m


def attend(state, seen, q, k, v, n_new, trees=None, softcap=0.0, slopes=None, window=0, sinks=0, p_half_step=0.0):
    """q [L, T, Hq, d], k, v [L, T, Hkv, d] (device tensors); seen[b]: tokens seen before the chunk; trees: (parents, depths) or None (a line).
    Returns out, its tolerance, mass, its tolerance (dicts by slab), rows (dict: K, V, pos)."""
    c = state.c
    L, T, Hq, d = q.shape
    G = Hq // c.kv_heads
    kv8 = c.dtype_name == "bf16_kv8"
    out = torch.zeros((L, T, Hq, d), dtype=torch.float64)
    tol = torch.zeros_like(out)
    mass, mass_tol, rows = {}, {}, {}
    for l in range(L):
        first = 0
        for b in range(c.batch):
            t = int(n_new[b])
            mine = slice(first, first + t)
            first += t
            for h in range(c.kv_heads):
                K, V, pos, _ = state.slab[l, b, h]
                kn, vn = k[l, mine, h].cpu(), v[l, mine, h].cpu()
                if kv8:
                    kn, vn = e4m3(kn, state.scales[0]).double() * state.scales[0], e4m3(vn, state.scales[1]).double() * state.scales[1]
                n = K.shape[0]
                K, V = torch.cat([K, kn.double()]), torch.cat([V, vn.double()])
                step = torch.tensor(trees[1][b], dtype=torch.long) if trees else torch.arange(t)
                pos = torch.cat([pos, seen[b] + step])
                rows[l, b, h] = (K, V, pos)
                if t == 0:
                    continue
                fresh = ancestors(trees[0][b]) if trees else torch.ones((t, t), dtype=torch.bool).tril()
                visible = torch.cat([torch.ones((t, n), dtype=torch.bool), fresh], 1)
                apart = (pos[n:, None] - pos[None, :]).abs()
                if window:
                    visible &= (apart < window) | (pos < sinks)[None]
                m, mt = torch.zeros(n + t, dtype=torch.float64), torch.zeros(n + t, dtype=torch.float64)
                for x in range(h * G, (h + 1) * G):
                    qx = q[l, mine, x].cpu().double()
                    z = qx @ K.T / math.sqrt(d)
                    dz = (d + 8) * 2.0 ** -23 * (qx.abs() @ K.abs().T) / math.sqrt(d) + 8 * 2.0 ** -24 * z.abs()
                    if softcap:
                        z = softcap * torch.tanh(z / softcap)
                        dz = dz + 16 * 2.0 ** -24 * softcap
                    if slopes is not None:
                        bias = float(slopes[x]) * apart
                        z = z - bias
                        dz = dz + 8 * 2.0 ** -24 * bias
                    dz = dz + 8 * 2.0 ** -24 * z.abs()
                    z = z.masked_fill(~visible, -math.inf)
                    dz = dz.masked_fill(~visible, 0.0).amax(-1, keepdim=True)
                    p = torch.softmax(z, -1)
                    rel = 2 * dz + (2 * 2 + 128) * 2.0 ** -23
                    Vx = V.masked_fill(~visible.any(0)[:, None], 0.0)  # (rows nobody sees may hold anything)
                    o, mag = p @ Vx, p @ Vx.abs()
                    out[l, mine, x] = o
                    tol[l, mine, x] = (rel + p_half_step + (n + t) / 8 * 2.0 ** -23) * mag * 1.01 + EPS[q.dtype] * o.abs() * 1.01 + 1e-30
                    m += p.sum(0)
                    mt += (p * rel).sum(0)
                mass[l, b, h] = m
                mass_tol[l, b, h] = mt * 1.01 + (t * G + 8) * 2.0 ** -24 * m + 1e-30
    return out, tol, mass, mass_tol, rows


def sample(logits, u, temperature, top_k, top_p, min_p):
    """One token and log-probability per row, the settings as the 32-bit values a call is given (lists or numbers)."""
    n, V = logits.shape
    f32 = lambda x: float(torch.tensor(x, dtype=torch.float32))
    per = lambda x: x.tolist() if hasattr(x, "tolist") else list(x) if isinstance(x, (list, tuple)) else [x] * n
    T, k, p, low = per(temperature), per(top_k), per(top_p), per(min_p)
    tokens, logprobs = [], []
    for r in range(n):
        x = logits[r].double().cpu()
        if torch.isnan(x).any() or x.max() == math.inf or x.max() == -math.inf:
            tokens.append(-1)
            logprobs.append(math.nan)
            continue
        order = torch.sort(x, descending=True, stable=True).indices
        if not f32(T[r]) > 0:
            tokens.append(int(order[0]))
            logprobs.append(0.0)
            continue
        w = torch.exp((x - x.max()) / f32(T[r]))
        keep = order[: k[r]] if k[r] > 0 else order
        if f32(p[r]) < 1:
            s = w[keep].cumsum(0)
            keep = keep[: max(1, int((torch.cat([torch.zeros(1, dtype=torch.float64), s[:-1]]) < f32(p[r]) * s[-1]).sum()))]
        keep = keep[(w[keep] >= min(f32(low[r]), 1.0)) | (w[keep] == 1.0)]
        keep = keep.sort().values
        s = w[keep].cumsum(0)
        uu = float(u[r])
        uu = min(uu, 1 - 2.0 ** -24) if uu >= 0 else 0.0
        at = int((s <= uu * s[-1]).sum())
        last = int((w[keep] > 0).nonzero().max())
        at = min(at, last)
        tokens.append(int(keep[at]))
        logprobs.append(float((w[keep[at]] / s[-1]).log()))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(logprobs, dtype=torch.float64)
