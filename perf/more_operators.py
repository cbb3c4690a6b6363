"""Checking drafted trees, sampling the answers, and windows with sinks, as cases to measure: what each reads, its
plain form in elementary torch operations, its definition in 64 bits, and the calls a user makes of the library.

  tree     a tree of drafted tokens per sequence (parents before children) against the rows the cache holds: the
           tree is numbered, its rows are stored behind the sequence's end, every node attends to the sequence's
           rows, to its ancestors in the tree and to itself; its position is the tokens seen plus its depth
  sinks    a chunk of tokens (one per sequence, or many) that sees a sliding window of positions and the first few
           positions of its sequence, which stay visible whatever the window
  sample   a token per row of logits: temperature, top-k, top-p and min-p, from a given random number
  verify   the same for every node of drafted trees, and the path of nodes whose tokens were drawn

The cases use the attention shapes of this repository's workloads: 32 query / 8 KV heads, 28 / 4 heads, and the tiny
fp32 configuration; rows of 16 bits, of 8 bits with a scale, and of 32 bits; vocabularies from 1000 to 152064.
"""
import math
import random

import torch

own = False

KV_SCALE = 0.05  # scale of the 8-bit rows: the planted keys reach about 12, the format 448 * 0.05 = 22


def _case(name, kind, **kw):
    case = dict(kind=kind)
    if kind in ("tree", "sinks"):
        case.update(batch=1, q_heads=32, kv_heads=8, d=128, rows="bf16", past_lo=0, past_hi=0, new_lo=1, new_hi=1, softcap=0.0, bias=False, window=0,
                    sinks=0, depth=8, roots=1, mass=False, deal=1)
    else:
        case.update(rows=1, vocab=128256, dtype="bf16", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, spread=2.0, batch=1, new_lo=1,
                    new_hi=1, depth=8, roots=1, deal=1)
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # checking a small drafted tree of one sequence against a cache at its budget: latency
        _case("tree of 12 over 2048", "tree", past_lo=2048, past_hi=2048, new_lo=12, new_hi=12, depth=4),
        # a serving batch: ragged trees behind ragged caches
        _case("trees 32 x 25 ragged", "tree", batch=32, q_heads=28, kv_heads=4, past_lo=900, past_hi=2111, new_lo=9, new_hi=25, depth=6, deal=5),
        # 8-bit rows, the widest trees that are usual, long caches
        _case("trees 8-bit 16 x 60 over 4200", "tree", batch=16, q_heads=28, kv_heads=4, rows="kv8", past_lo=4100, past_hi=4224, new_lo=60, new_hi=60, depth=7, deal=6),
        # the tiny fp32 configuration, an odd tree, and the importance its nodes give the rows
        _case("tree fp32 d64 41 over 131", "tree", q_heads=4, kv_heads=1, d=64, rows="fp32", past_lo=131, past_hi=131, new_lo=41, new_hi=41, mass=True),
        # one decode step of a ragged batch of 64 long sequences in a model with a window and sinks
        _case("sinks step 64 over 4200", "sinks", batch=64, past_lo=3000, past_hi=4223, window=1024, sinks=4, deal=7),
        # further questions, capped logits, a short window: ragged
        _case("sinks turns 8 capped", "sinks", batch=8, q_heads=28, kv_heads=4, past_lo=1500, past_hi=6000, new_lo=17, new_hi=700, window=511, sinks=16, softcap=50.0, deal=9),
        # a long prompt read in one call
        _case("sinks prompt 8000", "sinks", new_lo=8000, new_hi=8000, window=1024, sinks=4),
        # one sequence's next token: latency
        _case("sample 1 x 128256", "sample", temperature=0.7, top_k=50, top_p=0.9),
        # a serving batch, each row with its own settings, 32-bit logits
        _case("sample 64 x 152064 mixed", "sample", rows=64, vocab=152064, dtype="fp32", mixed=True),
        # many samples of flat distributions, nothing cut: the whole vocabulary counts; an odd vocabulary
        _case("sample 256 x 50257 uncut", "sample", rows=256, vocab=50257, dtype="fp32", temperature=1.3, spread=2.5),
        # the nodes of one tree
        _case("verify 1 x 60", "verify", new_lo=60, new_hi=60, temperature=0.8, top_p=0.95, depth=7),
        # the nodes of a serving batch's trees
        _case("verify 32 x 25", "verify", batch=32, new_lo=25, new_hi=25, temperature=0.6, top_k=200, top_p=0.95, min_p=0.01, depth=6),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "sinks", "sinks", "sample", "sample", "verify"])
    deal = rng.randrange(1, 1 << 20)
    if kind in ("sample", "verify"):
        case = _case(None, kind, vocab=rng.choice([128256, 152064, _log_int(rng, 1000, 150000)]), dtype=rng.choice(["bf16", "fp32"]),
                     temperature=rng.choice([0.0, 0.6, 0.8, 1.0, 1.4]), spread=rng.choice([1.5, 2.0, 2.5]), deal=deal, depth=rng.choice([3, 5, 8]))
        which = rng.randrange(0, 8)
        if which & 1:
            case["top_k"] = _log_int(rng, 1, 2000)
        if which & 2:
            case["top_p"] = rng.choice([0.5, 0.8, 0.9, 0.95, 0.99])
        if which & 4:
            case["min_p"] = rng.choice([0.005, 0.05, 0.1])
        case["mixed"] = rng.random() < 0.3
        room = 30000000 // case["vocab"]
        if kind == "sample":
            case["rows"] = _log_int(rng, 1, min(300, room))
        else:
            case["batch"] = rng.choice([1, 2, 7, 16])
            case["new_hi"] = _log_int(rng, 2, min(64, room // case["batch"]))
            case["new_lo"] = rng.choice([case["new_hi"], 1])
        return case
    q_heads, kv_heads = rng.choice([(32, 8), (28, 4)])
    rows = rng.choice(["bf16", "bf16", "kv8", "fp32"])
    most = 64 if kind == "tree" else 4000
    if rows == "fp32":  # small: head sizes other than 128, as in the tiny configuration
        past = _log_int(rng, 8, 500)
        case = _case(None, kind, batch=rng.choice([1, 2, 3]), q_heads=4, kv_heads=rng.choice([1, 2]), d=rng.choice([64, 64, 40]), rows=rng.choice(["fp32", "fp32", "bf16"]),
                     past_lo=past // 2, past_hi=past, new_lo=1, new_hi=_log_int(rng, 1, 60), deal=deal)
    else:
        batch = rng.choice([1, 2, 5, 16, 33])
        past = _log_int(rng, 16, min(6000, 60000 // batch))
        new = _log_int(rng, 1, max(2, min(most, 4000 // batch)))
        if kind == "sinks" and rng.random() < 0.4:
            new = 1
        case = _case(None, kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, rows=rows, past_lo=rng.choice([past, past // 2, past // 8]), past_hi=past,
                     new_lo=rng.choice([new, max(1, new // 3), 1]), new_hi=new, deal=deal)
    if kind == "tree":
        case["depth"], case["roots"], case["mass"] = rng.choice([2, 4, 6, 9]), rng.choice([1, 1, 3]), rng.random() < 0.3
    else:
        case["window"], case["sinks"], case["mass"] = _log_int(rng, 8, 3000), _log_int(rng, 1, 80), rng.random() < 0.2
    which = rng.randrange(0, 8)
    if which == 1:
        case["softcap"] = rng.choice([20.0, 30.0, 50.0])
    if which == 2:
        case["bias"] = True
    return case


def _lengths(case):
    """Rows held and tokens brought by every sequence."""
    r = random.Random(case["deal"])
    past = [r.randint(case.get("past_lo", 0), case.get("past_hi", 0)) for _ in range(case["batch"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    return past, new


def _trees(case, new, seed):
    """Parents (-1: none) and depths of every sequence's nodes, level by level as a drafting model grows them."""
    r = random.Random(case["deal"] * 1000003 + seed)
    parents, depths = [], []
    for n in new:
        p, dep = [], []
        for i in range(n):
            if i < min(case["roots"], n):
                p.append(-1)
                dep.append(0)
                continue
            lo = max(0, i - 1 - r.choice([0, 2, 8, 30]))  # nodes grow from recent ones for the most part
            up = r.randint(lo, i - 1)
            while dep[up] + 1 >= case["depth"]:
                up = p[up]
            p.append(up)
            dep.append(dep[up] + 1)
        parents.append(p)
        depths.append(dep)
    return parents, depths


def _settings(case, n, g):
    """Temperature, top_k, top_p and min_p of every row: tensors where the rows differ."""
    if not case["mixed"]:
        return dict(temperature=case["temperature"], top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])

    def pick(values, dtype):
        at = torch.randint(0, len(values), (n,), generator=g, device="cuda")
        return torch.tensor(values, dtype=dtype, device="cuda")[at]

    return dict(temperature=pick([0.0, 0.5, 0.7, 1.0, 1.0, 1.2], torch.float32), top_k=pick([0, 0, 20, 50, 400], torch.int32),
                top_p=pick([1.0, 0.9, 0.95, 0.8], torch.float32), min_p=pick([0.0, 0.0, 0.05, 0.1], torch.float32))


def _prepare_logits(case, seed, g):
    _, new = _lengths(case)
    verify = case["kind"] == "verify"
    n, V = (sum(new) if verify else case["rows"]), case["vocab"]
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    # the bulk of a vocabulary, and a few dozen tokens that the model considers
    x = torch.randn((n, V), generator=g, device="cuda") * case["spread"]
    few = torch.randint(0, V, (n, 40), generator=g, device="cuda")
    lift = 4.0 + 3.0 * torch.empty((n, 40), device="cuda").exponential_(1.0, generator=g)
    x.scatter_(1, few, lift.clamp(max=25.0))
    s = dict(case=case, logits=x.to(dt), u=torch.rand((n,), generator=g, device="cuda"))
    s["settings"] = _settings(case, n, g)
    s["tokens"] = torch.empty((n,), dtype=torch.int32, device="cuda")
    s["logprobs"] = torch.empty((n,), device="cuda")
    if verify:
        parents, _ = _trees(case, new, seed)
        first = [sum(new[:b]) for b in range(len(new))]
        r = random.Random(seed * 31 + case["deal"])
        pick = [r.choice([0, 0, 0, 1, 2, 5]) for _ in range(n)]
        best = x.topk(6, dim=1).indices  # a draft proposes what its parent's distribution favours
        flat = [f + max(p, 0) for f, ps in zip(first, parents) for p in ps]
        s["drafted"] = best[torch.tensor(flat, device="cuda"), torch.tensor(pick, device="cuda")].int()
        s["parents"] = torch.tensor([p for ps in parents for p in ps], dtype=torch.int32, device="cuda")
        s["n_new"] = torch.tensor(new, dtype=torch.int32)
        s["seq"] = torch.repeat_interleave(torch.arange(len(new), device="cuda"), torch.tensor(new, device="cuda"))
        s["first"] = torch.tensor(first, device="cuda")
        s["path"] = torch.empty((len(new), case["depth"]), dtype=torch.int32, device="cuda")
        s["accepted"] = torch.empty((len(new),), dtype=torch.int32, device="cuda")
        s["next"] = torch.empty((len(new),), dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)
    if case["kind"] in ("sample", "verify"):
        return _prepare_logits(case, seed, g)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    dt = torch.float32 if case["rows"] == "fp32" else torch.bfloat16
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
    s["out"] = torch.empty_like(s["q"])
    s["mass"] = torch.zeros((1, nb, hkv, cap), device="cuda") if case["mass"] else None
    if case["kind"] == "tree":
        parents, _ = _trees(case, new, seed)
        s["parents"] = torch.tensor([p for ps in parents for p in ps], dtype=torch.int32, device="cuda")
        s["tree"] = torch.empty((total, 4), dtype=torch.int32, device="cuda")
        s["positions"] = torch.empty((total,), dtype=torch.int32, device="cuda")
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
    kind = case["kind"]
    if not own:
        return {"tree": _plain_attention, "sinks": _plain_attention, "sample": _plain_sample, "verify": _plain_verify}[kind](s)
    import paper_2601_18383_b200 as D
    if kind in ("sample", "verify"):
        D.sample(s["logits"], s["u"], tokens=s["tokens"], logprobs=s["logprobs"], **s["settings"])
        if kind == "sample":
            return s["tokens"], s["logprobs"]
        D.tree_accept(s["parents"], s["drafted"], s["tokens"], s["n_new"], path=s["path"], accepted=s["accepted"], next_tokens=s["next"])
        return s["tokens"], s["logprobs"], s["path"], s["accepted"], s["next"]
    c = s["cache"]
    options = dict(softcap=case["softcap"], slopes=s["slopes"], mass=s["mass"], stage=True)
    # staged: the rows are stored behind the end, the sequences' lengths stay (a draft that is checked)
    if kind == "tree":
        c.tree_plan(s["parents"], s["n_new"], tree=s["tree"], positions=s["positions"])
        c.extend_attn_layer(0, s["q"], s["k"], s["v"], s["out"], s["n_new"], tree=s["tree"], **options)
    else:
        c.extend_attn_layer(0, s["q"], s["k"], s["v"], s["out"], s["n_new"], window=case["window"], sinks=case["sinks"], **options)
    outs = [s["out"]]
    if case["mass"]:
        outs.append(s["mass"])
    if kind == "tree":
        outs.append(s["positions"])
    return outs


def _plain_attention(s):
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
    row = torch.arange(cap, device="cuda")
    # positions are the tokens seen before: row j of a sequence that lost none is position j
    pos = row.expand(nb, cap)
    if case["kind"] == "tree":
        first = torch.zeros_like(past).scatter_reduce(0, seq, torch.arange(seq.numel(), device="cuda"), "amin", include_self=False)
        above = s["parents"].long()
        mine = torch.zeros((nb, tm, tm), dtype=torch.bool, device="cuda")  # node i sees node j
        depth, up = torch.zeros_like(off), off.clone()
        for _ in range(case["depth"]):
            mine[seq, off, up.clamp(min=0)] |= up >= 0
            up = torch.where(up >= 0, above[first[seq] + up.clamp(min=0)], up)
            depth += (up >= 0).long()
        me = torch.zeros((nb, tm), dtype=torch.long, device="cuda")
        me[seq, off] = past[seq] + depth
        pos = pos.clone()
        pos[seq, at] = past[seq] + depth
        at_node = (row - past[:, None]).clamp(0, tm - 1)  # [nb, cap]
        fresh = (row >= past[:, None]) & (row < (past + torch.bincount(seq, minlength=nb))[:, None])
        seen = (row < past[:, None])[:, None] | (fresh[:, None] & mine.gather(2, at_node[:, None].expand(nb, tm, cap)))
    else:
        me = past[:, None] + torch.arange(tm, device="cuda")  # [nb, tm]
        seen = row <= me[..., None]
    apart = (me[..., None] - pos[:, None]).abs()  # [nb, tm, cap]
    if case["window"]:
        seen = seen & ((apart < case["window"]) | (pos < case["sinks"])[:, None])
    real = torch.zeros((nb, tm), dtype=torch.bool, device="cuda")
    real[seq, off] = True
    S = torch.matmul(q.reshape(nb, hkv, G * tm, d), K.transpose(-1, -2)).reshape(nb, hkv, G, tm, cap) / math.sqrt(d)
    if case["softcap"]:
        S = case["softcap"] * torch.tanh(S / case["softcap"])
    if case["bias"]:
        S = S - s["slopes"].reshape(1, hkv, G, 1, 1) * apart[:, None, None].float()
    S = S.masked_fill(~seen[:, None, None], float("-inf"))
    P = torch.exp(S - S.amax(-1, keepdim=True))
    P = P / P.sum(-1, keepdim=True)
    P = P.masked_fill(~real[:, None, None, :, None], 0.0)  # (places of a batch that hold no token)
    O = torch.matmul(P.reshape(nb, hkv, G * tm, cap), V).reshape(nb, hkv, G, tm, d)
    outs = [O.permute(0, 3, 1, 2, 4)[seq, off].reshape(-1, hq, d).to(s["q"].dtype)]
    if case["mass"]:
        outs.append(P.sum((2, 3))[None])
    if case["kind"] == "tree":
        outs.append((past[seq] + depth).int())
    return outs


def _row(value, n, dtype):
    """A setting of every row, as 64-bit values of what the call is given."""
    if not torch.is_tensor(value):
        value = torch.full((n,), value, dtype=dtype, device="cuda")
    return (value.double() if dtype is torch.float32 else value.long())[:, None]


def _plain_sample(s):
    # 64 bits: sums over a whole vocabulary, and values next to a border
    x = s["logits"].double()
    n, V = x.shape
    t, p, low = (_row(s["settings"][k], n, torch.float32) for k in ("temperature", "top_p", "min_p"))
    k = _row(s["settings"]["top_k"], n, torch.int32)
    greedy = t <= 0
    top = x.amax(-1, keepdim=True)
    w = torch.exp((x - top) / torch.where(greedy, 1.0, t))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    rank = torch.arange(V, device="cuda")[None]
    keep = (rank < torch.where(k > 0, k, V))
    ws = ws * keep
    run_up = ws.cumsum(-1)
    before = torch.cat([torch.zeros_like(run_up[:, :1]), run_up[:, :-1]], -1)
    keep &= (p >= 1) | (before < p * run_up[:, -1:])
    keep &= ws >= low
    keep |= rank == 0
    wi = w * torch.zeros_like(keep).scatter(1, order, keep)
    cdf = wi.cumsum(-1)
    total = cdf[:, -1:]
    at = (cdf <= s["u"].double()[:, None] * total).sum(-1, keepdim=True)
    last = torch.where(wi > 0, rank, -1).amax(-1, keepdim=True)
    at = torch.minimum(at, last)
    logprob = torch.log(wi.gather(1, at) / total)
    best = torch.where(x == top, rank, V).amin(-1, keepdim=True)
    at, logprob = torch.where(greedy, best, at), torch.where(greedy, 0.0, logprob)
    return at[:, 0].int(), logprob[:, 0].float()


def _plain_verify(s):
    tokens, logprobs = _plain_sample(s)
    first, seq = s["first"], s["seq"]
    nb, n = first.numel(), seq.numel()
    index = torch.arange(n, device="cuda")
    at = first.clone()  # the node each sequence's path has reached: its first, to begin with
    alive = torch.ones_like(first, dtype=torch.bool)
    path, accepted = [torch.zeros_like(first)], torch.ones_like(first)
    parent = torch.where(s["parents"] < 0, -1, s["parents"].long() + first[seq])
    for _ in range(s["case"]["depth"] - 1):
        fits = (parent == at[seq]) & (s["drafted"] == tokens[at][seq]) & alive[seq]
        child = torch.full((nb,), n, device="cuda").scatter_reduce(0, seq, torch.where(fits, index, n), "amin")
        alive = child < n
        at = torch.where(alive, child, at)
        accepted = accepted + alive.long()
        path.append(torch.where(alive, child - first, -1))
    return tokens, logprobs, torch.stack(path, 1).int(), accepted.int(), tokens[at]


def work(case):
    past, new = _lengths(case)
    if case["kind"] in ("sample", "verify"):
        n = sum(new) if case["kind"] == "verify" else case["rows"]
        # the logits, the random numbers, the tokens and their log-probabilities; a scaled difference, an exponential and a sum each
        return {"bytes": n * (case["vocab"] * (4 if case["dtype"] == "fp32" else 2) + 12), "flops": 4 * n * case["vocab"]}
    hq, hkv, d, w, x = case["q_heads"], case["kv_heads"], case["d"], case["window"], case["sinks"]
    size = 4 if case["rows"] == "fp32" else 2
    row = {"fp32": 4, "bf16": 2, "kv8": 1}[case["rows"]] * d
    pairs = held = 0
    _, depths = _trees(case, new, 0) if case["kind"] == "tree" else (None, None)
    for b, (n, t) in enumerate(zip(past, new)):
        if case["kind"] == "tree":
            pairs += n * t + sum(i + 1 for i in depths[b])
            held += n
            continue
        for i in range(t):
            me = n + i
            lo = max(0, me - w + 1)
            pairs += me - lo + 1 + min(x, lo)
        lo = max(0, n - w + 1)
        held += min(n, n - lo + min(x, lo))
    tokens = sum(new)
    # the queries, the output, the new rows read and stored, the rows held; the mass of every row, the parents and positions
    moved = 2 * tokens * hq * d * size + 2 * tokens * hkv * (d * size + row) + 2 * held * hkv * row
    if case["mass"]:
        moved += 4 * hkv * (sum(past) + tokens)
    if case["kind"] == "tree":
        moved += 8 * tokens
    return {"bytes": moved, "flops": 4 * pairs * hq * d}


def exact(case, seed):
    """From the definitions, in 64 bits: one sequence and KV head, or one row of logits, at a time."""
    s = prepare(case, seed)
    past, new = _lengths(case)
    if case["kind"] in ("sample", "verify"):
        return _exact_sample(case, s, new)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["d"]
    G = hq // hkv
    value = (lambda x: x.double() * KV_SCALE) if case["rows"] == "kv8" else (lambda x: x.double())
    fresh = _codes if case["rows"] == "kv8" else (lambda x: x)
    out = torch.empty((sum(new), hq, d), dtype=torch.float64, device="cuda")
    mass = torch.zeros((1, case["batch"], hkv, s["cap"]), dtype=torch.float64, device="cuda")
    positions = []
    parents, depths = _trees(case, new, seed) if case["kind"] == "tree" else (None, None)
    start = 0
    for b, (n, t) in enumerate(zip(past, new)):
        mine = slice(start, start + t)
        start += t
        place = list(range(n)) + ([n + x for x in depths[b]] if parents else list(range(n, n + t)))
        positions += place[n:]
        place = torch.tensor(place, device="cuda")
        distance = (place[n:, None] - place[None, :]).abs()
        if parents:
            visible = torch.zeros((t, n + t), dtype=torch.bool)
            visible[:, :n] = True
            for i in range(t):
                j = i
                while j >= 0:
                    visible[i, n + j] = True
                    j = parents[b][j]
            visible = visible.cuda()
        else:
            visible = torch.ones((t, n + t), dtype=torch.bool, device="cuda").tril(n)
            visible &= (distance < case["window"]) | (place < case["sinks"])[None]
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
    outs = [out]
    if case["mass"]:
        outs.append(mass)
    if parents:
        outs.append(torch.tensor(positions, dtype=torch.int32, device="cuda"))
    return outs


def _exact_sample(case, s, new):
    n = s["logits"].shape[0]
    if n * case["vocab"] > 150000000:
        return None
    setting = {k: (v.tolist() if torch.is_tensor(v) else torch.tensor([v], dtype=torch.int32 if k == "top_k" else torch.float32).tolist() * n)
               for k, v in s["settings"].items()}
    tokens, logprobs = [], []
    for r in range(n):
        x = s["logits"][r].double()
        values, order = x.sort(descending=True, stable=True)
        t = setting["temperature"][r]
        if t <= 0:
            tokens.append(order[0])
            logprobs.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        w = ((values - values[0]) / t).exp()
        if setting["top_k"][r] > 0:
            w = w[: setting["top_k"][r]]
        if setting["top_p"][r] < 1:  # the shortest run of the largest that reaches p
            reached = torch.searchsorted(w.cumsum(0), setting["top_p"][r] * w.sum())
            w = w[: int(reached) + 1]
        w = w[w >= setting["min_p"][r]] if setting["min_p"][r] < 1 else w[w >= 1]
        kept, back = order[: w.numel()].sort()
        line = w[back].cumsum(0)
        at = torch.searchsorted(line, s["u"][r].double() * line[-1], right=True).clamp(max=w.numel() - 1)
        tokens.append(kept[at])
        logprobs.append((w[back][at] / line[-1]).log())
    tokens, logprobs = torch.stack(tokens).int(), torch.stack(logprobs)
    if case["kind"] == "sample":
        return tokens, logprobs
    drawn, drafted, parents = tokens.tolist(), s["drafted"].tolist(), s["parents"].tolist()
    paths, counts, ends, start = [], [], [], 0
    for t in new:
        path = [0]
        while len(path) < case["depth"]:
            fit = [i for i in range(t) if parents[start + i] == path[-1] and drafted[start + i] == drawn[start + path[-1]]]
            if not fit:
                break
            path.append(fit[0])
        paths.append(path + [-1] * (case["depth"] - len(path)))
        counts.append(len(path))
        ends.append(drawn[start + path[-1]])
        start += t
    whole = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return tokens, logprobs, whole(paths), whole(counts), whole(ends)
