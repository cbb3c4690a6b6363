"""Trees, sampling, accepted paths and windows with sinks used together: a small model whose answers are drawn token by token, and the
same answers found by checking drafted trees."""
import math

import pytest
import torch

import paper_2601_18383_b200 as D

pytestmark = pytest.mark.gpu

L, HQ, HKV, HD, HID, VOCAB, BATCH = 2, 4, 2, 64, 96, 211, 3


class Small:
    def __init__(self, seed, dtype=torch.float32, d=HD):
        g = torch.Generator(device="cuda").manual_seed(seed)
        mk = lambda *s: torch.randn(s, generator=g, device="cuda") / math.sqrt(s[-1])
        self.embed, self.head = mk(VOCAB, HID) * math.sqrt(HID), mk(VOCAB, HID) * 6.0
        self.w = [dict(q=mk(HQ * d, HID), k=mk(HKV * d, HID), v=mk(HKV * d, HID), o=mk(HID, HQ * d)) for _ in range(L)]
        self.dtype, self.d = dtype, d

    def logits(self, cache, tokens, pos, n_new, **opt):
        x = self.embed[tokens.long()]
        n = tokens.numel()
        for l, w in enumerate(self.w):
            q, k, v = ((x @ w[m].T).to(self.dtype).view(n, -1, self.d) for m in "qkv")
            q, k = D.rope(q, k, pos, theta=1000.0)
            out = torch.empty_like(q)
            cache.extend_attn_layer(l, q.contiguous(), k.contiguous(), v.contiguous(), out, n_new, **opt)
            x = x + out.float().view(n, -1) @ w["o"].T
        return x @ self.head.T

    def cache(self, name):
        return D.Cache(L, BATCH, HQ, HKV, self.d, 200, 8, 56, dtype=name)


def one_by_one(model, cache, prompts, u, steps, settings, opt):
    """Prompt, then a token per step: token s of sequence b is drawn with u[b, s]."""
    n_new = [len(p) for p in prompts]
    pos = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in n_new])
    x = model.logits(cache, torch.cat(prompts), pos, n_new, **opt)
    last = torch.tensor([sum(n_new[: b + 1]) - 1 for b in range(BATCH)], device="cuda")
    answer = [D.sample(x[last].contiguous(), u[:, 0].contiguous(), **settings)[0]]
    for s in range(1, steps):
        pos = torch.tensor([n + s - 1 for n in n_new], device="cuda", dtype=torch.int32)
        x = model.logits(cache, answer[-1], pos, [1] * BATCH, **opt)
        answer.append(D.sample(x, u[:, s].contiguous(), **settings)[0])
    return torch.stack(answer, 1)


def by_trees(model, cache, prompts, u, steps, settings, opt, guess):
    """The same by checking trees: node 0 is the token drawn last; guess(b, s, node) proposes tokens for step s."""
    n_new = [len(p) for p in prompts]
    pos = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in n_new])
    x = model.logits(cache, torch.cat(prompts), pos, n_new, **opt)
    at = torch.tensor([sum(n_new[: b + 1]) - 1 for b in range(BATCH)], device="cuda")
    answer = [[t] for t in D.sample(x[at].contiguous(), u[:, 0].contiguous(), **settings)[0].tolist()]
    checks = 0
    while min(len(a) for a in answer) < steps:
        tokens, parents, chance, counts = [], [], [], []
        for b in range(BATCH):
            done = len(answer[b])
            t, p, depth = [answer[b][-1]], [-1], [0]
            if done < steps:
                for node in range(6):  # the first nodes get children
                    if node >= len(t) or depth[node] >= 3:
                        continue
                    for y in guess(b, done + depth[node], node):
                        t.append(y), p.append(node), depth.append(depth[node] + 1)
            else:
                t, p, depth = [], [], []
            tokens += t
            parents += p
            chance += [float(u[b, min(done + x, steps - 1)]) for x in depth]
            counts.append(len(t))
        up = torch.tensor(parents, dtype=torch.int32, device="cuda")
        tree, pos = cache.tree_plan(up, counts)
        flat = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        x = model.logits(cache, flat, pos, counts, tree=tree, stage=True, **opt)
        drawn, _ = D.sample(x, torch.tensor(chance, device="cuda"), **settings)
        path, accepted, ends = D.tree_accept(up, flat, drawn, counts, 4)
        cache.extend_commit_path(accepted.tolist(), path)
        first = 0
        for b in range(BATCH):
            on = [i for i in path[b].tolist() if i >= 0]
            answer[b] += [tokens[first + i] for i in on[1:]] + ([int(ends[b])] if on else [])
            first += counts[b]
        checks += 1
    cache.poll_error()
    return torch.tensor([a[:steps] for a in answer]), checks


@pytest.mark.parametrize("opt", [dict(), dict(window=20, sinks=3), dict(softcap=20.0)], ids=["plain", "sinks", "cap"])
@pytest.mark.parametrize("settings", [dict(temperature=0.0), dict(temperature=0.8, top_k=30, top_p=0.95), dict(temperature=1.2, min_p=0.02)], ids=["greedy", "top", "min"])
def test_checked_trees_give_the_answers_of_single_steps(settings, opt):
    """fp32: a row's logits differ by rounding between the two, and the random numbers are the same ones."""
    model = Small(3)
    g = torch.Generator(device="cuda").manual_seed(5)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g, device="cuda") for n in (30, 1, 17)]
    u = torch.rand((BATCH, 40), generator=g, device="cuda")
    steps = 40
    a = model.cache("fp32")
    want = one_by_one(model, a, prompts, u, steps, settings, opt).cpu()
    a.close()
    r = torch.Generator().manual_seed(9)

    def guess(b, s, node):  # often right
        right = int(want[b, min(s, steps - 1)])
        wrong = [int(y) for y in torch.randint(0, VOCAB, (2,), generator=r)]
        return [wrong[0], right] if torch.rand((), generator=r) < 0.7 else wrong

    c = model.cache("fp32")
    got, checks = by_trees(model, c, prompts, u, steps, settings, opt, guess)
    c.close()
    assert torch.equal(got, want.long())
    assert checks < steps - 1


def test_trees_and_steps_at_head_size_128():
    """bf16 rows: the small-chunk kernel, the tensor-core kernel and the commit on one cache; every node's logits against the line's."""
    model = Small(4, torch.bfloat16, 128)
    c = model.cache("bf16")
    g = torch.Generator(device="cuda").manual_seed(5)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g, device="cuda") for n in (60, 70, 50)]
    pos = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in (60, 70, 50)])
    model.logits(c, torch.cat(prompts), pos, [60, 70, 50])
    line = torch.randint(0, VOCAB, (BATCH, 40), generator=g, device="cuda")
    parents = torch.arange(-1, 39, dtype=torch.int32, device="cuda").repeat(BATCH)
    tree, pos = c.tree_plan(parents, [40] * BATCH)
    far = model.logits(c, line.reshape(-1), pos, [40] * BATCH, tree=tree, stage=True)   # 80 query rows: tensor cores
    near = []
    for s in range(0, 40, 5):
        pos = torch.cat([n + torch.arange(s, s + 5, device="cuda", dtype=torch.int32) for n in (60, 70, 50)])
        near.append(model.logits(c, line[:, s:s + 5].reshape(-1), pos, [5] * BATCH).view(BATCH, 5, VOCAB))  # 10 query rows
    c.poll_error()
    near = torch.cat(near, 1).reshape(-1, VOCAB)
    assert [c.len(b) for b in range(BATCH)] == [100, 110, 90]
    # outputs of two layers, rounded to bf16 (2^-8) from weights rounded to bf16: a few 2^-8 of a logit's size, 6
    assert (far - near).abs().max() < 16 * 2.0 ** -8 * 6
    c.close()
