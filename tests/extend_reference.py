"""Plain 64-bit forms of the chunk operators, and how far a kernel may be from them by its roundings.

The reference takes what the cache held before the chunk (exported slabs) and the chunk itself, and
returns per layer the outputs, the rows' attention mass, and a bound for each output's error."""
import math

import torch

EPS = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # a rounding's largest relative error: half a step


def e4m3(x, scale):
    """Codes of a float tensor: value(code nearest to x / scale), ties to even, saturating."""
    return (x.float() / scale).clamp(-448, 448).to(torch.float8_e4m3fn)


class State:
    """What a cache holds, as 64-bit values on the host: K, V, pos, score per (layer, sequence, KV head)."""

    def __init__(self, cache, k_scale=1.0, v_scale=1.0):
        self.c, self.scales = cache, (k_scale, v_scale)
        self.slab = {}
        for l in range(cache.layers):
            for b in range(cache.batch):
                for h in range(cache.kv_heads):
                    K, V, pos, score = cache.export_slab(l, b, h)
                    self.slab[l, b, h] = [self.value(K, k_scale), self.value(V, v_scale), pos.long(), score.double()]

    @staticmethod
    def value(x, scale):
        return x.view(torch.float8_e4m3fn).double() * scale if x.dtype == torch.uint8 else x.double()


def extend(state, seen, q, k, v, n_new, softcap=0.0, slopes=None, window=0, prefix=None, p_half_step=0.0):
    """q [L, T, Hq, d], k, v [L, T, Hkv, d] (device tensors); seen[b]: tokens seen by sequence b before the chunk.

    p_half_step: relative half step of the type the kernel rounds its weights to before it multiplies them with V
    (0: they stay fp32).  Returns out, mass (dict by slab), tol (as out), mass_tol (as mass), rows (dict: K, V, pos)."""
    c = state.c
    L, T, Hq, d = q.shape
    G = Hq // c.kv_heads
    kv8 = c.dtype_name == "bf16_kv8"
    out = torch.zeros((L, T, Hq, d), dtype=torch.float64)
    tol = torch.zeros_like(out)
    mass, mass_tol, rows = {}, {}, {}
    eps_out = EPS[q.dtype]
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
                K, V = torch.cat([K, kn.double()]), torch.cat([V, vn.double()])
                pos = torch.cat([pos, seen[b] + torch.arange(t)])
                rows[l, b, h] = (K, V, pos)
                if t == 0:
                    continue
                n = K.shape[0] - t
                i, j = torch.arange(t)[:, None], torch.arange(n + t)[None, :]
                visible = j < n + torch.clamp(i + 1, min=int(prefix[b]) if prefix is not None else 0)
                apart = (pos[n:, None] - pos[None, :]).abs()
                if window:
                    visible &= apart < window
                m, mt = torch.zeros(n + t, dtype=torch.float64), torch.zeros(n + t, dtype=torch.float64)
                for x in range(h * G, (h + 1) * G):
                    qx = q[l, mine, x].cpu().double()
                    z = qx @ K.T / math.sqrt(d)
                    # an fp32 dot product of d terms, summed in any order, is off by at most d half steps of the sum of
                    # magnitudes; the tensor cores may cut instead of rounding (a whole step).  Scaling, cap, bias and the
                    # change to base 2 add a few half steps of the values they handle.
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
                    # every weight is off by at most 2 dz (its own logit's error and the sum's), the exponentials' own error
                    # (2 steps each), and the sum of the weights by a half step per term of its longest chain (<= 64 + log)
                    rel = 2 * dz + (2 * 2 + 128) * 2.0 ** -23
                    o = p @ V
                    mag = p @ V.abs()
                    out[l, mine, x] = o
                    # weights rounded before the product, the product's fp32 accumulation (a step per 16 keys), the output
                    tol[l, mine, x] = (rel + p_half_step + (n + t) / 8 * 2.0 ** -23) * mag * 1.01 + eps_out * o.abs() * 1.01 + 1e-30
                    m += p.sum(0)
                    mt += (p * rel).sum(0)
                mass[l, b, h] = m
                # a column's sum of t * G weights in fp32
                mass_tol[l, b, h] = mt * 1.01 + (t * G + 8) * 2.0 ** -24 * m + 1e-30
    return out, mass, tol, mass_tol, rows
