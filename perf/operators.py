"""Operators around the budget-limited cache, as cases to measure: what each reads, its plain form in
elementary torch operations, its definition in 64 bits, and the call a user makes of the library.

  chunk    a chunk of new tokens per sequence (ragged) against the rows the cache holds: the rows are
           stored behind the sequence's end, every token attends to the sequence's rows and to the
           chunk up to itself
  variant  the same with logits capped by a tanh, a bias that falls with the distance, a window of
           positions, and a prefix of the chunk that every token of the chunk sees
  mass     the same, and the attention mass every row received from the chunk's queries (the importance
           a selection ranks rows by)
  rope     rotary positions with one or several axes, on the queries and keys of a batch of tokens

The cases use the attention shapes of this repository's workloads: 32 query / 8 KV heads, 28 / 4 heads,
and the tiny fp32 configuration; rows of 16 bits, of 8 bits with a scale, and of 32 bits.
"""
import math
import random

import torch

own = False

KV_SCALE = 0.05  # scale of the 8-bit rows: the planted keys reach about 12, the format 448 * 0.05 = 22
THETA = 500000.0


def _attn(name, kind, **kw):
    case = dict(kind=kind, batch=1, q_heads=32, kv_heads=8, d=128, rows="bf16", past_lo=0, past_hi=0, new_lo=1, new_hi=1,
                softcap=0.0, bias=False, window=0, prefix=0, deal=1)
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _rope(name, **kw):
    case = dict(kind="rope", tokens=1, q_heads=32, kv_heads=8, d=128, rot=128, axes=1, dtype="bf16", pairs="half", far=32768)
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # checking five drafted tokens of one sequence against a cache at its budget: latency
        _attn("verify 5 over 2048", "chunk", past_lo=2048, past_hi=2048, new_lo=5, new_hi=5),
        # the next turn of sixteen conversations: ragged questions behind ragged caches
        _attn("turns 16 ragged", "chunk", batch=16, q_heads=28, kv_heads=4, past_lo=900, past_hi=4224, new_lo=17, new_hi=390, deal=5),
        # a long document read in pieces: the second piece of 4096 tokens
        _attn("piece 4096 over 4096", "chunk", past_lo=4096, past_hi=4096, new_lo=4096, new_hi=4096),
        # 8-bit rows: a short follow-up to sixteen long sequences, bound by the rows it reads
        _attn("8-bit 16 x 12 over 4200", "chunk", batch=16, q_heads=28, kv_heads=4, rows="kv8", past_lo=4100, past_hi=4224, new_lo=12, new_hi=12, deal=6),
        # the tiny fp32 configuration, an odd chunk
        _attn("fp32 d64 48 over 131", "chunk", q_heads=4, kv_heads=1, d=64, rows="fp32", past_lo=131, past_hi=131, new_lo=48, new_hi=48),
        # one decode step of a ragged batch of 64 in a model with capped logits and a sliding window
        _attn("step 64 capped window", "variant", batch=64, past_lo=1000, past_hi=2111, new_lo=1, new_hi=1, softcap=50.0, window=1024, deal=7),
        # ragged prompts packed one after another into an empty cache, with a distance bias
        _attn("packed prompts bias", "variant", batch=8, past_lo=0, past_hi=0, new_lo=33, new_hi=1100, bias=True, deal=8),
        # a prompt whose first part (an image, a system text) is seen by all of it, capped logits, behind a cache
        _attn("prefix 700 of 1500 capped", "variant", batch=2, q_heads=28, kv_heads=4, past_lo=513, past_hi=777, new_lo=1500, new_hi=1500, softcap=30.0, prefix=700, deal=9),
        # the importance a question of 200 tokens gives the rows of a cache at its budget
        _attn("mass 200 over 2112", "mass", past_lo=2112, past_hi=2112, new_lo=200, new_hi=200),
        # the same for a ragged batch with long questions
        _attn("mass 4 ragged long", "mass", batch=4, q_heads=28, kv_heads=4, past_lo=2000, past_hi=6000, new_lo=300, new_hi=2000, deal=10),
        # one decode step of 16 sequences: latency
        _rope("rotate step 16", tokens=16, q_heads=28, kv_heads=4),
        # a prompt with images: three axes, 16384 tokens
        _rope("rotate 16384 three axes", tokens=16384, axes=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunk", "chunk", "variant", "variant", "mass", "rope"])
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4)])
    if kind == "rope":
        d = rng.choice([128, 128, 64])
        rot = rng.choice([d, d, d // 2])
        return _rope(None, tokens=_log_int(rng, 1, 8000), q_heads=q_heads, kv_heads=kv_heads, d=d, rot=rot, axes=rng.choice([1, 2, 3, 3]),
                     dtype=rng.choice(["bf16", "bf16", "fp32"]), pairs=rng.choice(["half", "half", "adjacent"]), far=_log_int(rng, 4096, 1000000))
    rows = rng.choice(["bf16", "bf16", "kv8", "fp32"])
    deal = rng.randrange(1, 1 << 20)
    if rows == "fp32":  # small: head sizes other than 128, as in the tiny configuration
        past, new = _log_int(rng, 8, 500), _log_int(rng, 1, 96)
        case = _attn(None, kind, batch=rng.choice([1, 2, 3]), q_heads=4, kv_heads=rng.choice([1, 2]), d=rng.choice([64, 64, 40]), rows=rng.choice(["fp32", "fp32", "bf16"]),
                     past_lo=past // 2, past_hi=past, new_lo=1, new_hi=new, deal=deal)
    else:
        batch = rng.choice([1, 2, 5, 16, 33])
        past = _log_int(rng, 16, min(6000, 30000 // batch))
        new = _log_int(rng, 1, max(2, 4000 // batch))
        case = _attn(None, kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, rows=rows, past_lo=rng.choice([past, past // 2, past // 8]),
                     past_hi=past, new_lo=rng.choice([new, max(1, new // 3), 1]), new_hi=new, deal=deal)
    if kind == "variant" or (kind == "mass" and rng.random() < 0.4):
        which = rng.randrange(1, 16)
        if which & 1:
            case["softcap"] = rng.choice([20.0, 30.0, 50.0])
        if which & 2:
            case["bias"] = True
        if which & 4:
            case["window"] = _log_int(rng, 16, 4000)
        if which & 8:
            case["prefix"] = _log_int(rng, 1, case["new_hi"])
    return case


def _lengths(case):
    """Rows held and tokens brought by every sequence."""
    r = random.Random(case["deal"])
    past = [r.randint(case["past_lo"], case["past_hi"]) for _ in range(case["batch"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    return past, new


def _sections(case):
    half, axes = case["rot"] // 2, case["axes"]
    rest = (half // axes) // 2 * 2 if axes > 1 else half
    return [half - rest * (axes - 1)] + [rest] * (axes - 1)


def _dtype(case):
    return torch.float32 if case.get("rows", case.get("dtype")) == "fp32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    dt = _dtype(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if case["kind"] == "rope":
        n = case["tokens"]
        s = dict(case=case, q=normal(n, case["q_heads"], case["d"]).to(dt), k=normal(n, case["kv_heads"], case["d"]).to(dt))
        s["pos"] = torch.randint(0, case["far"], (case["axes"], n), generator=g, device="cuda", dtype=torch.int32)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["sections"] = _sections(case)
        return s
    past, new = _lengths(case)
    nb, hq, hkv, d = case["batch"], case["q_heads"], case["kv_heads"], case["d"]
    total, cap = sum(new), max(p + t for p, t in zip(past, new))
    cap = (cap + 31) // 32 * 32
    # one row in twenty carries the direction its head's queries look for, as in the planted workloads
    a = math.sqrt(4.0 * math.sqrt(d))
    u = normal(nb, hkv, d)
    u = u / u.norm(dim=-1, keepdim=True)
    seq = torch.repeat_interleave(torch.arange(nb, device="cuda"), torch.tensor(new, device="cuda"))
    first = torch.tensor([sum(new[:b]) for b in range(nb)], device="cuda")
    off = torch.arange(total, device="cuda") - first[seq]

    def crit(*shape):
        return a * (torch.rand(shape, generator=g, device="cuda") < 0.05).float()[..., None]

    s = dict(case=case, past=torch.tensor(past, device="cuda"), seq=seq, off=off, cap=cap)
    s["q"] = (normal(total, hkv, hq // hkv, d) + a * u[seq][:, :, None]).to(dt).reshape(total, hq, d)
    s["k"] = (normal(total, hkv, d) + crit(total, hkv) * u[seq]).to(dt)
    s["v"] = normal(total, hkv, d).to(dt)
    K = (normal(nb, hkv, cap, d) + crit(nb, hkv, cap) * u[:, :, None]).to(dt)
    V = normal(nb, hkv, cap, d).to(dt)
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device="cuda") / hq) if case["bias"] else None
    s["n_new"] = torch.tensor(new, dtype=torch.int32)
    s["prefix"] = torch.tensor([min(case["prefix"], t) for t in new], dtype=torch.int32) if case["prefix"] else None
    s["prefix_dev"] = torch.tensor([min(case["prefix"], t) for t in new], device="cuda")
    s["out"] = torch.empty_like(s["q"])
    s["mass"] = torch.zeros((1, nb, hkv, cap), device="cuda") if case["kind"] == "mass" else None
    if own:
        import paper_2601_18383_b200 as D
        c = D.Cache(1, nb, hq, hkv, d, cap, 0, 1, dtype={"kv8": "bf16_kv8"}.get(case["rows"], case["rows"]), capacity=cap)
        if case["rows"] == "kv8":
            c.set_kv_scale(KV_SCALE, KV_SCALE)
        c.set_score_source(D.DYNTS_SCORE_EXTERNAL)
        for b in range(nb):
            if past[b]:
                c.prefill_seq(b, K[None, b, :, : past[b]].contiguous(), V[None, b, :, : past[b]].contiguous(), n_pinned=0)
        c.synchronize()
        s["cache"] = c
    else:  # the plain form's cache: the rows as they are stored
        s["K"], s["V"] = (_codes(K), _codes(V)) if case["rows"] == "kv8" else (K, V)
    return s


def _codes(x):
    return (x.float() / KV_SCALE).clamp(-448, 448).to(torch.float8_e4m3fn)


def run(s):
    case = s["case"]
    if case["kind"] == "rope":
        if own:
            import paper_2601_18383_b200 as D
            D.rope(s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], theta=THETA, sections=s["sections"], adjacent=case["pairs"] == "adjacent")
            return s["q_out"], s["k_out"]
        return _plain_rope(s)
    if own:
        # staged: the chunk's rows are stored behind the end, the sequences' lengths stay (a draft that is checked)
        s["cache"].extend_attn_layer(0, s["q"], s["k"], s["v"], s["out"], s["n_new"], mass=s["mass"], softcap=case["softcap"], slopes=s["slopes"],
                                     window=case["window"], prefix=s["prefix"], stage=True)
        return (s["out"], s["mass"]) if case["kind"] == "mass" else s["out"]
    return _plain_extend(s)


def _plain_rope(s):
    case = s["case"]
    half, d = case["rot"] // 2, case["d"]
    freq = THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(s["sections"], device="cuda"))
    angle = s["pos"].double()[axis].T * freq  # [tokens, half]: 64 bits, the angles of far positions
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotate(x):
        y = x.float()
        if case["pairs"] == "half":
            a, b = y[..., :half], y[..., half:2 * half]
            r = torch.cat([a * cos - b * sin, a * sin + b * cos, y[..., 2 * half:]], -1)
        else:
            a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
            r = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), y[..., 2 * half:]], -1)
        return r.to(x.dtype)

    return rotate(s["q"]), rotate(s["k"])


def _plain_extend(s):
    case, seq, off, past = s["case"], s["seq"], s["off"], s["past"]
    nb, hq, hkv, d = case["batch"], case["q_heads"], case["kv_heads"], case["d"]
    G, cap, tm = hq // hkv, s["cap"], case["new_hi"]
    K, V = s["K"], s["V"]
    k, v = s["k"], s["v"]
    if case["rows"] == "kv8":  # the new rows are stored in 8 bits too, and read as stored
        K, V, k, v = K.float() * KV_SCALE, V.float() * KV_SCALE, _codes(k).float() * KV_SCALE, _codes(v).float() * KV_SCALE
    K, V = K.float().clone(), V.float().clone()
    at = past[seq] + off
    K[seq, :, at], V[seq, :, at] = k.float(), v.float()
    q = torch.zeros((nb, tm, hkv, G, d), device="cuda")
    q[seq, off] = s["q"].float().reshape(-1, hkv, G, d)
    q = q.permute(0, 2, 3, 1, 4)  # [nb, hkv, G, tm, d]
    S = torch.matmul(q.reshape(nb, hkv, G * tm, d), K.transpose(-1, -2)).reshape(nb, hkv, G, tm, cap) / math.sqrt(d)
    if case["softcap"]:
        S = case["softcap"] * torch.tanh(S / case["softcap"])
    row = torch.arange(cap, device="cuda")
    # positions are the tokens seen before: row j of a sequence that lost none is position j
    me = past[:, None] + torch.arange(tm, device="cuda")  # [nb, tm]
    apart = (me[..., None] - row).abs()  # [nb, tm, cap]
    if case["bias"]:
        S = S - s["slopes"].reshape(1, hkv, G, 1, 1) * apart[:, None, None].float()
    seen = row <= me[..., None]
    if case["prefix"]:
        seen = seen | (row < (past + s["prefix_dev"])[:, None, None])
    if case["window"]:
        seen = seen & (apart < case["window"])
    S = S.masked_fill(~seen[:, None, None], float("-inf"))
    P = torch.exp(S - S.amax(-1, keepdim=True))
    P = P / P.sum(-1, keepdim=True)
    O = torch.matmul(P.reshape(nb, hkv, G * tm, cap), V).reshape(nb, hkv, G, tm, d)
    out = O.permute(0, 3, 1, 2, 4)[seq, off].reshape(-1, hq, d).to(s["q"].dtype)
    if case["kind"] != "mass":
        return out
    real = torch.zeros((nb, tm), device="cuda")
    real[seq, off] = 1.0
    return out, (P * real[:, None, None, :, None]).sum((2, 3))[None]


def work(case):
    if case["kind"] == "rope":
        size = 4 if case["dtype"] == "fp32" else 2
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["d"]
        return {"bytes": 2 * values * size + 4 * case["tokens"] * case["axes"], "flops": 3 * values}
    past, new = _lengths(case)
    hq, hkv, d, w = case["q_heads"], case["kv_heads"], case["d"], case["window"]
    size = 4 if case["rows"] == "fp32" else 2
    row = {"fp32": 4, "bf16": 2, "kv8": 1}[case["rows"]] * d
    pairs = held = 0
    for n, t in zip(past, new):
        x = min(case["prefix"], t)
        for i in range(t):  # rows that token i sees
            last = max(n + i, n + x - 1)
            lo, hi = (max(0, n + i - w + 1), min(last, n + i + w - 1)) if w else (0, last)
            pairs += hi - lo + 1
        held += n - max(0, n - w + 1) if w else n
    tokens = sum(new)
    # the queries, the output, the new rows read and stored, the rows held; the mass of every row where it is asked for
    moved = 2 * tokens * hq * d * size + 2 * tokens * hkv * (d * size + row) + 2 * held * hkv * row
    if case["kind"] == "mass":
        moved += 4 * hkv * (sum(past) + tokens)
    return {"bytes": moved, "flops": 4 * pairs * hq * d}


def exact(case, seed):
    """From the definitions, in 64 bits, one sequence and KV head at a time."""
    s = prepare(case, seed)
    if case["kind"] == "rope":
        half = case["rot"] // 2
        axis = [a for a, n in enumerate(s["sections"]) for _ in range(n)]
        turned = []
        for x in (s["q"], s["k"]):
            z = x.double()
            r = z.clone()
            for i in range(half):
                p, m = (i, i + half) if case["pairs"] == "half" else (2 * i, 2 * i + 1)
                phi = s["pos"][axis[i]].double()[:, None] * THETA ** (-2.0 * i / case["rot"])
                r[..., p] = z[..., p] * phi.cos() - z[..., m] * phi.sin()
                r[..., m] = z[..., p] * phi.sin() + z[..., m] * phi.cos()
            turned.append(r)
        return tuple(turned)
    past, new = _lengths(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["d"]
    G = hq // hkv
    value = (lambda x: x.double() * KV_SCALE) if case["rows"] == "kv8" else (lambda x: x.double())
    fresh = _codes if case["rows"] == "kv8" else (lambda x: x)
    out = torch.empty((sum(new), hq, d), dtype=torch.float64, device="cuda")
    mass = torch.zeros((1, case["batch"], hkv, s["cap"]), dtype=torch.float64, device="cuda")
    start = 0
    for b, (n, t) in enumerate(zip(past, new)):
        mine = slice(start, start + t)
        start += t
        i = torch.arange(t, device="cuda")[:, None]
        j = torch.arange(n + t, device="cuda")[None, :]
        visible = (j <= n + i) | (j < n + min(case["prefix"], t))
        distance = (n + i - j).abs()
        if case["window"]:
            visible &= distance < case["window"]
        for h in range(hkv):
            K = torch.cat([value(s["K"][b, h, :n]), value(fresh(s["k"][mine, h]))])
            V = torch.cat([value(s["V"][b, h, :n]), value(fresh(s["v"][mine, h]))])
            for x in range(h * G, (h + 1) * G):
                logit = s["q"][mine, x].double() @ K.T / d ** 0.5
                if case["softcap"]:
                    logit = case["softcap"] * (logit / case["softcap"]).tanh()
                if case["bias"]:
                    logit = logit - float(s["slopes"][x]) * distance
                weight = logit.masked_fill(~visible, -math.inf).softmax(-1)
                out[mine, x] = weight @ V
                mass[0, b, h, : n + t] += weight.sum(0)
    return (out, mass) if case["kind"] == "mass" else out
