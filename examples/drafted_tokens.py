"""Drafted tokens over pages, one attention layer: answers to one compressed prompt go on by trees of drafted tokens, of which those that the layer's head finds
probable are kept.

    prompt          hot_path (chunks, ranking, eviction) -> page_append: the kept keys and values, already rotated, into pages that all answers share
    a step          page_append (drafted keys and values, rotated by their depth in the tree) -> tree_attn (every drafted token over the prompt, the answer so far and its
                    ancestors) -> head -> token_logprobs (each drafted token under its parent's logits) -> the path that is kept -> page_append (pick, count)

The layer, its head and the drafts are random, so the answers mean nothing; pages, trees, positions and calls are those of a model's layer.  Chunks are ranked by
their self-information, the sum of the window's log probabilities behind each (token_logprobs with group).  At the end the last step is computed again in plain PyTorch from a
record of what was kept, without the pages.

    python examples/drafted_tokens.py [--answers 4] [--steps 6] [--format bf16|int8|e4m3]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_14317_b200 as pc  # noqa: E402

I32 = torch.int32
# two guesses for the next token, two behind each, one more behind the first two of those
PARENTS = [-1, -1, 0, 0, 1, 1, 2, 3]


def rotate(x, pos, theta):
    """rotate-half RoPE of x [n,H,d] at positions pos [n], in 64 bits"""
    d = x.shape[-1]
    angle = pos.double().unsqueeze(-1) * theta ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    c, s = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1)
    a, b = x.double().split(d // 2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Layer:
    def __init__(self, vocabulary, Hq, Hkv, d, seed):
        self.Hq, self.Hkv, self.d = Hq, Hkv, d
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda n, m, s: (torch.randn(n, m, generator=g, device="cuda") * s).to(torch.bfloat16)          # noqa: E731
        width = Hq * d
        self.embed, self.qkv = make(vocabulary, width, 1.0), make(width, (Hq + 2 * Hkv) * d, width ** -0.5)
        self.out, self.head = make(width, width, width ** -0.5), make(width, vocabulary, 3.0 * width ** -0.5)

    def project(self, x):
        """x [B,n,Hq*d] -> q, k, v [B,n,H,d], unrotated"""
        y = (x @ self.qkv).view(*x.shape[:2], -1, self.d)
        return y[:, :, :self.Hq], y[:, :, self.Hq:self.Hq + self.Hkv], y[:, :, self.Hq + self.Hkv:]

    def logits(self, attended):
        """attended [B,n,Hq,d] -> [B,n,V]"""
        y = attended.flatten(2) @ self.out
        return (y / y.float().pow(2).mean(-1, keepdim=True).sqrt().clamp_min(1e-6).to(y.dtype)) @ self.head


def kept_path(logprob, parents, least):
    """The drafted tokens that are kept of a sequence: from the context's end always the most probable child, as long as it is probable enough"""
    path, at = [], -1
    while True:
        children = [i for i, p in enumerate(parents) if p == at and logprob[i] > least]
        if not children:
            return path
        at = max(children, key=lambda i: logprob[i])
        path.append(at)


def run(answers=4, steps=6, fmt="bf16", *, chunks=6, chunk_len=1024, w=32, Hq=16, Hkv=4, d=128, theta=5e5, m=3, k_keep=256, page=32, vocabulary=5000, least=-9.0,
        seed=0):
    layer, g = Layer(vocabulary, Hq, Hkv, d, seed), torch.Generator(device="cuda").manual_seed(seed + 1)
    tokens = torch.randint(0, vocabulary, (chunks, chunk_len), generator=g, device="cuda")
    tokens[:, -w:] = tokens[:1, -w:]                                      # every chunk ends with the same query window

    # the prompt: the window's log probabilities behind each chunk rank the chunks
    q, k, v = (t.contiguous() for t in layer.project(layer.embed[tokens]))
    pre = pc.chunk_prefill_attn(q, k, v, w=w, rope_theta=theta)
    window = layer.logits(pre["o"][:, -w - 1:-1]).flatten(0, 1)           # the token before each of the window's
    score = pc.token_logprobs(window, tokens[:, -w:].flatten().to(I32), group=w)["nll"]
    res = pc.hot_path(q, k, v, w=w, rope_theta=theta, m=m, k_keep=k_keep, chunk_score=score)
    last = layer.logits(res["fg"])[:, -1].expand(answers, -1).contiguous()

    # pages: the prompt's first, shared; then each answer's own
    n_prompt, depth, n_tree = m * k_keep, max(len(p) for p in _paths(PARENTS)), len(PARENTS)
    assert n_prompt % page == 0
    shared, own = n_prompt // page, -(-(steps * depth + n_tree) // page)
    pool = pc.kv_cache(shared + answers * own, Hkv, page, d, fmt)
    table = torch.cat([torch.arange(shared, device="cuda").expand(answers, -1),
                       shared + torch.randperm(answers * own, generator=g, device="cuda").view(answers, own)], 1).to(I32).contiguous()
    pc.page_append(pool, res["kc"].transpose(0, 1).unsqueeze(0), res["vc"].transpose(0, 1).unsqueeze(0), table[:1], at=0)
    lens = torch.full((answers,), n_prompt, dtype=I32, device="cuda")
    pos = torch.full((answers,), chunk_len, dtype=I32, device="cuda")     # the answers go on where the window ended
    parents, status, buffers = torch.tensor(PARENTS, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda"), {}
    each = parents.expand(answers, -1)
    record = [[] for _ in range(answers)]                                 # what was kept: (key, value, position), unrotated

    for step in range(steps):
        drafts = torch.randint(0, vocabulary, (answers, n_tree), generator=g, device="cuda", dtype=I32)
        drafts[:, 0] = last.argmax(-1).to(I32)                            # a guess that holds
        q, k, v = layer.project(layer.embed[drafts.long()])
        pc.page_append(pool, k, v, table, at=lens, pos=pos, parents=each, rope_theta=theta, status=status)
        got = pc.tree_attn(q, pool, table, lens, parents=parents, pos=pos, rope_theta=theta, want_lse=True, buffers=buffers)
        logits = layer.logits(got["out"])
        above = torch.cat([last.unsqueeze(1), logits], 1)[:, [p + 1 for p in PARENTS]]
        logprob = pc.token_logprobs(above.flatten(0, 1), drafts.flatten(), top=4)["logprob"].view(answers, n_tree)
        if step == steps - 1:
            break
        paths = [kept_path(row, PARENTS, least) for row in logprob.tolist()]
        pick = torch.tensor([p + [-1] * (depth - len(p)) for p in paths], dtype=I32, device="cuda")
        count = torch.tensor([len(p) for p in paths], dtype=I32, device="cuda")
        pc.page_append(pool, k, v, table, at=lens, pos=pos, pick=pick, count=count, rope_theta=theta, status=status)
        for b, path in enumerate(paths):
            record[b] += [(k[b, i], v[b, i], int(pos[b]) + j) for j, i in enumerate(path)]
            if path:
                last[b] = logits[b, path[-1]]
        lens += count
        pos += count
    assert status.item() == 0 and got["status"].item() == 0

    # the last step again, from the record
    off = size = 0.0
    seen = _paths(PARENTS)
    for b in range(answers):
        keys = [res["kc"].double().transpose(0, 1)] + [rotate(x.unsqueeze(0), torch.tensor([p], device="cuda"), theta) for x, _, p in record[b]]
        values = [res["vc"].double().transpose(0, 1)] + [x.double().unsqueeze(0) for _, x, _ in record[b]]
        at = torch.tensor([int(pos[b]) + len(s) - 1 for s in seen], device="cuda")
        keys, values = torch.cat(keys + [rotate(k[b], at, theta)]), torch.cat(values + [v[b].double()])
        hidden = torch.ones(n_tree, len(keys), dtype=torch.bool, device="cuda")
        hidden[:, :len(keys) - n_tree] = False
        for i, s in enumerate(seen):
            hidden[i, [len(keys) - n_tree + j for j in s]] = False
        G = Hq // Hkv
        z = torch.einsum("ihgd,nhd->hgin", rotate(q[b], at, theta).view(n_tree, Hkv, G, d), keys) * d ** -0.5
        want = torch.einsum("hgin,nhd->ihgd", z.masked_fill(hidden, -torch.inf).softmax(-1), values).reshape(n_tree, Hq, d)
        off, size = max(off, (got["out"][b].double() - want).abs().max().item()), max(size, want.abs().max().item())
    return {"relative_difference": off / size, "kept": [len(r) for r in record], "entries": lens.tolist(), "chunk_score": score.tolist(), "chunks": res["kept"].tolist()}


def _paths(parents):
    paths = []
    for i, p in enumerate(parents):
        paths.append((paths[p] if p >= 0 else []) + [i])
    return paths


if __name__ == "__main__":
    args = argparse.ArgumentParser(description="Drafted tokens over the pages of a compressed prompt")
    args.add_argument("--answers", type=int, default=4)
    args.add_argument("--steps", type=int, default=6)
    args.add_argument("--format", choices=("bf16", "int8", "e4m3"), default="bf16")
    a = args.parse_args()
    r = run(a.answers, a.steps, a.format)
    print("%d answers: %s tokens kept in %d steps; entries %s; last step off by %.1e of its largest value" %
          (a.answers, r["kept"], a.steps - 1, r["entries"], r["relative_difference"]))
