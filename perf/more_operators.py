"""Performance cases of paged caches, of attention for drafted tokens over them, and of log probabilities.

Kinds of work (field ``kind``):
  append   ``page_append``: keys, rotated to their positions on the way, and values of new tokens go into the pages of their sequences; the whole
           pool of pages is returned (8-bit pages as the values that they stand for)
  tree     ``tree_attn``: w drafted tokens of B sequences, each the child of an earlier one, attend to their sequence's pages and to their own ancestors
  logprob  ``token_logprobs``: log probabilities of given tokens, the entropy, the most probable alternatives, and sums over groups of rows

Inputs follow the distributions that the repository's tests and benchmark draw: N(0,1) queries, keys and values and an attention
sink, with a few channels of the keys several times larger than the others, as keys have them; pages lie in the pool in no order, and what stands
behind a sequence's end is what an earlier one left there.
"""
import math

import torch

own = False
DEV = "cuda"
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
TOP = {"int8": 127.0, "e4m3": 448.0}                     # largest code of a format
TINY = 2.0 ** -100                                       # rows below it are stored as zeros


def _append(name, B, n, Hkv, d, fmt, page, theta, at, how="plain", fused=False, far=0):
    """at: entries that are there before (the most, where how is not "plain").  how: "plain"; "tree": drafted tokens, rotated by their depth, fewer of them
    in some sequences; "accept": up to n of 4 n drafted tokens, those that were accepted.  fused: slices of one projection.  far: added to positions"""
    return {"name": name, "kind": "append", "B": B, "n": n, "Hkv": Hkv, "d": d, "fmt": fmt, "page": page, "theta": theta, "at": at, "how": how,
            "fused": fused, "far": far}


def _tree(name, B, w, Hq, Hkv, d, fmt, page, theta, n, ragged, drafted):
    """n: entries before the new tokens, ragged: of different lengths; drafted: the tokens are a tree (else each sees all before it)"""
    return {"name": name, "kind": "tree", "B": B, "w": w, "Hq": Hq, "Hkv": Hkv, "d": d, "fmt": fmt, "page": page, "theta": theta, "n": n,
            "ragged": ragged, "drafted": drafted}


def _logprob(name, N, V, type, top, group, pad=0):
    """pad: elements between the rows"""
    return {"name": name, "kind": "logprob", "N": N, "V": V, "type": type, "top": top, "group": group, "pad": pad}


def listed():
    return [
        # the new token of one sequence: latency
        _append("append-token", 1, 1, 8, 128, "bf16", 64, 5.0e5, 1000),
        # drafts of 16 tokens of 23 sequences into small 8-bit pages, out of a fused projection, small heads
        _append("append-drafts-d64", 23, 16, 2, 64, "e4m3", 16, 1.0e6, 300, "tree", True),
        # what was accepted of 64 sequences' drafts, 8 bits
        _append("append-accepted-b64", 64, 5, 8, 128, "int8", 32, 5.0e5, 200, "accept"),
        # the keys and values of a 64K prompt, positions that fp32 angles do not reach
        _append("append-prompt-64k", 1, 65537, 8, 128, "bf16", 128, 5.0e5, 0, far=100000),
        # one generation step of one sequence: latency
        _tree("token-b1", 1, 1, 32, 8, 128, "bf16", 64, 5.0e5, 16400, False, False),
        # one generation step of 64 sequences of different lengths in 8 bits: the memory's rate
        _tree("token-b64-int8", 64, 1, 32, 8, 128, "int8", 32, 5.0e5, 16384, True, False),
        # drafts of 12 tokens of 23 sequences, 84 rows per kv-head, small heads, small pages
        _tree("drafts-b23-d64", 23, 12, 14, 2, 64, "bf16", 16, 1.0e6, 5000, True, True),
        # a tree of 64 drafted tokens over one long context: 256 rows per kv-head
        _tree("tree64-b1", 1, 64, 32, 8, 128, "bf16", 128, 5.0e5, 32768, False, True),
        # trees of 40 tokens of 16 sequences: the matrix units' rate
        _tree("tree40-b16", 16, 40, 32, 8, 128, "bf16", 64, 5.0e5, 12000, True, True),
        # the next token of one sequence with 20 alternatives: latency
        _logprob("logprob-token", 1, 128256, "fp32", 20, 0),
        # drafted tokens to be verified, rows that begin anywhere
        _logprob("logprob-drafts-odd", 276, 50001, "fp16", 5, 0, 2),
        # the query window behind each of 16 chunks: the chunks' self-information
        _logprob("logprob-chunks", 1024, 128256, "bf16", 8, 64),
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))

    largest = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["append", "tree", "tree", "logprob"])
        d, Hkv, page, theta = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 48, 64, 128, 256]), rng.choice([1.0e4, 5.0e5, 1.0e6])
        fmt = rng.choice(["bf16", "bf16", "int8", "e4m3"])
        if kind == "append":
            how = rng.choice(["plain", "plain", "tree", "accept"])
            n = spread(1, 65536) if how == "plain" else spread(1, 64 if how == "tree" else 16)
            c = _append("", spread(1, 64), n, Hkv, d, fmt, page, theta, spread(1, 1000), how, rng.random() < 0.5, rng.choice([0, 0, 70000]))
        elif kind == "tree":
            w = spread(1, 64)
            c = _tree("", spread(1, 64), w, rng.choice([1, 2, 3, 4, 7, 8]) * Hkv, Hkv, d, fmt, page, theta, spread(1, 40000), rng.random() < 0.5,
                      w > 1 and rng.random() < 0.7)
        else:
            group = rng.choice([0, 0, 8, 64])
            N = spread(1, 2000) if group == 0 else group * spread(1, 2000 // group)
            c = _logprob("", N, spread(1000, 200000), rng.choice(["bf16", "fp16", "fp32"]), rng.choice([0, 1, 5, 20, 32]), group, rng.choice([0, 0, 1, 8]))
        del c["name"]
        if _cost(c) <= largest:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.4e15)


def _row(fmt, d):
    """bytes of an entry of one head, keys or values"""
    return 2 * d if fmt == "bf16" else d + 4


def _lens(c):
    """entries that the sequences have before"""
    most = c["at"] if c["kind"] == "append" else c["n"]
    if c["how"] == "plain" if c["kind"] == "append" else not c["ragged"]:
        return [most] * c["B"]
    return [(most * ((37 * b + 11) % 101)) // 100 for b in range(c["B"])]


def _pages(c):
    """pages of the longest sequence, and of the pool"""
    most = -(-((c["at"] if c["kind"] == "append" else c["n"]) + (c["n"] if c["kind"] == "append" else c["w"])) // c["page"])
    return most, c["B"] * most + 3


def work(case):
    c = case
    if c["kind"] == "logprob":
        rows = c["N"] * (4 + 4 + 4 + 8 * c["top"]) + (4 * c["N"] // c["group"] if c["group"] else 0)
        return {"bytes": c["N"] * c["V"] * TYPES[c["type"]].itemsize + rows, "flops": 5 * c["N"] * c["V"]}
    Hkv, d, q = c["Hkv"], c["d"], _row(c["fmt"], c["d"])
    if c["kind"] == "append":
        entries = 2 * Hkv * c["B"] * c["n"]
        back = 2 * Hkv * _pages(c)[1] * c["page"] * (q + 2 * d) if c["fmt"] != "bf16" else 0        # the pool, read back as values
        return {"bytes": entries * (2 * d + q) + back, "flops": 0}
    lens, rows = _lens(c), c["B"] * c["w"] * c["Hq"]
    keys = sum(lens) + c["B"] * c["w"]
    return {"bytes": Hkv * 2 * keys * q + 4 * rows * d + 4 * rows, "flops": 4 * c["Hq"] * c["w"] * d * (sum(lens) + c["B"])}


# ------------------------------------------------------------------------------------ inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=F32)


def _keys(gen, *shape):
    """keys [..., d]: N(0,1) with every 16th channel four times as large"""
    k = _normal(gen, *shape)
    k[..., ::16] *= 4.0
    return k.to(BF16)


def _scaled(x, fmt):
    """rows of x in 8 bits: codes and scales"""
    x = x.to(F32)
    a = x.abs().amax(-1)
    held = (a >= TINY) & torch.isfinite(a)
    r = torch.where(held, TOP[fmt] / a, torch.zeros_like(a))
    y = x * r.unsqueeze(-1)
    codes = torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
    scale = torch.where(held, a / TOP[fmt], torch.zeros_like(a))
    return codes, torch.where(torch.isfinite(a), scale, torch.full_like(a, math.nan))


def _values(codes, scale):
    """what a cache stands for, fp32"""
    return codes.to(F32) if scale is None else codes.to(F32) * scale.unsqueeze(-1)


def _pool(c, gen, filled):
    """a pool of pages [n_pages,Hkv,page,d] as a program has it, and the sequences' tables"""
    most, n = _pages(c)
    shape, fmt = (n, c["Hkv"], c["page"], c["d"]), c["fmt"]
    k, v = (torch.zeros(shape, device=DEV, dtype=torch.int8).view(CODES[fmt]) if fmt != "bf16" else torch.zeros(shape, device=DEV, dtype=BF16)
            for _ in range(2))
    ks, vs = (None, None) if fmt == "bf16" else (torch.zeros(shape[:3], device=DEV), torch.zeros(shape[:3], device=DEV))
    if filled:
        for i in range(0, n, 512):
            x, y = _keys(gen, min(512, n - i), *shape[1:]), _normal(gen, min(512, n - i), *shape[1:]).to(BF16)
            if fmt == "bf16":
                k[i:i + 512], v[i:i + 512] = x, y
            else:
                (k[i:i + 512], ks[i:i + 512]), (v[i:i + 512], vs[i:i + 512]) = _scaled(x, fmt), _scaled(y, fmt)
    table = torch.randperm(n, generator=gen, device=DEV)[:c["B"] * most].view(c["B"], most).to(I32)
    return {"format": fmt, "k": k, "v": v, "k_scale": ks, "v_scale": vs}, table


def _parents(gen, B, w, fewer):
    """trees: a token's parent is one of the four before it, or the context's end (-1); fewer: some have not all tokens (-2)"""
    i = torch.arange(w, device=DEV)
    back = torch.randint(1, 5, (B, w), generator=gen, device=DEV)
    p = (i - back).clamp(min=-1)
    if fewer:
        there = torch.randint((w + 1) // 2, w + 1, (B, 1), generator=gen, device=DEV)
        p = torch.where(i < there, p, torch.full_like(p, -2))
    return p.to(I32).contiguous()


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 23)
    s = {"case": c}
    if c["kind"] == "logprob":
        N, V = c["N"], c["V"]
        rows = torch.empty((N, V + c["pad"]), device=DEV, dtype=TYPES[c["type"]])
        for i in range(0, N, 256):
            x = _normal(gen, min(256, N - i), V + c["pad"]) * 2.5
            x[:, :V] += 6.0 * (torch.rand((x.shape[0], V), generator=gen, device=DEV) < 4.0 / V)         # a few that stand out
            rows[i:i + 256] = x.to(rows.dtype)
        s["logits"] = rows[:, :V]
        s["tokens"] = torch.where(torch.rand(N, generator=gen, device=DEV) < 0.5, s["logits"].argmax(-1),
                                  torch.randint(0, V, (N,), generator=gen, device=DEV)).to(I32)
        return s
    B, Hkv, d = c["B"], c["Hkv"], c["d"]
    s["lens"] = torch.tensor(_lens(c), device=DEV, dtype=I32)
    s["cache"], s["table"] = _pool(c, gen, c["kind"] == "tree")
    if c["kind"] == "append":
        n = 4 * c["n"] if c["how"] == "accept" else c["n"]
        if c["fused"]:
            both = _keys(gen, B, n, 6 * Hkv, d)
            s["k"], s["v"] = both[:, :, 4 * Hkv:5 * Hkv], both[:, :, 5 * Hkv:]
        else:
            s["k"], s["v"] = _keys(gen, B, n, Hkv, d), _normal(gen, B, n, Hkv, d).to(BF16)
        s["parents"] = _parents(gen, B, n, True) if c["how"] == "tree" else None
        s["pick"] = s["count"] = None
        if c["how"] == "accept":
            s["pick"] = torch.rand((B, n), generator=gen, device=DEV).topk(c["n"], -1).indices.sort(-1).values.to(I32).contiguous()
            s["count"] = torch.randint(0, c["n"] + 1, (B,), generator=gen, device=DEV, dtype=I32)
        return s
    s["q"] = _normal(gen, B, c["w"], c["Hq"], d).to(BF16)
    s["parents"] = _parents(gen, B, c["w"], True) if c["drafted"] else None
    s["keep"] = {}                                        # outputs and workspaces, kept from call to call
    return s


# ------------------------------------------------------------------------------------ plain form
def _ancestors(parents):
    """[B,w,w]: 1 where a token sees another, itself among them; rows of tokens that are not there: 0"""
    B, w = parents.shape
    there = parents >= -1
    a = (parents.unsqueeze(-1) == torch.arange(w, device=DEV)).to(F32) + torch.eye(w, device=DEV)
    a = (a @ a).clamp(max=1.0)                            # steps of up to 2, 4, .. 64
    a = (a @ a).clamp(max=1.0)
    a = (a @ a).clamp(max=1.0)
    a = (a @ a).clamp(max=1.0)
    a = (a @ a).clamp(max=1.0)
    a = (a @ a).clamp(max=1.0)
    return a * there.unsqueeze(-1)


def _rotate(x, pos, theta):
    """x [B,n,H,d] turned by its positions [B,n] (pairs (t, t + d/2)), fp32, angles in 64 bits"""
    d = x.shape[-1]
    a = pos.to(F64).unsqueeze(-1) * theta ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=F64) / d)
    co, si = torch.cos(a).to(F32).unsqueeze(2), torch.sin(a).to(F32).unsqueeze(2)
    u, v = x[..., :d // 2].to(F32), x[..., d // 2:].to(F32)
    return torch.cat([u * co - v * si, v * co + u * si], -1)


def _plain_append(s):
    c, cache = s["case"], s["cache"]
    B, n, page = c["B"], c["n"], c["page"]
    j = torch.arange(n, device=DEV).expand(B, n)
    k, v, step, there = s["k"], s["v"], j, None
    if s["parents"] is not None:
        step = _ancestors(s["parents"]).sum(-1).to(torch.int64) - 1
        there = step >= 0
    if s["pick"] is not None:
        b = torch.arange(B, device=DEV).unsqueeze(-1)
        k, v, there = k[b, s["pick"].long()], v[b, s["pick"].long()], j < s["count"].unsqueeze(-1)
    k = _rotate(k, s["lens"].unsqueeze(-1) + step + c["far"], c["theta"])
    entry = s["lens"].long().unsqueeze(-1) + j
    at = s["table"].long().gather(1, entry // page) * page + entry % page                # place in the pool
    written = lambda x: x.flatten(0, 1) if there is None else x[there]                   # noqa: E731
    at = written(at)

    def store(pool, x):                                                                  # pool [n_pages,Hkv,page,...], x [tokens,Hkv,...]
        pool.transpose(1, 2)[at // page, at % page] = x

    if c["fmt"] == "bf16":
        store(cache["k"], written(k).to(BF16))
        store(cache["v"], written(v))
        return {"k": cache["k"], "v": cache["v"]}
    (kc, ks), (vc, vs) = _scaled(written(k), c["fmt"]), _scaled(written(v), c["fmt"])
    store(cache["k"].view(torch.int8), kc.view(torch.int8))
    store(cache["v"].view(torch.int8), vc.view(torch.int8))
    store(cache["k_scale"], ks)
    store(cache["v_scale"], vs)
    return {"k": _values(cache["k"], cache["k_scale"]).to(BF16), "v": _values(cache["v"], cache["v_scale"]).to(BF16),
            "k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}


def _plain_tree(s):
    c = s["case"]
    B, w, Hq, Hkv, d, page = c["B"], c["w"], c["Hq"], c["Hkv"], c["d"], c["page"]
    G, lens = Hq // Hkv, s["lens"].long()
    if s["parents"] is None:
        sees = torch.ones((w, w), device=DEV).tril().expand(B, w, w)
    else:
        sees = _ancestors(s["parents"])
    depth = (sees.sum(-1) - 1).clamp(min=0)
    q = _rotate(s["q"], lens.unsqueeze(-1) + depth, c["theta"]).to(BF16).to(F32) / math.sqrt(d)
    q = q.view(B, w, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, w * G, d)
    entry = torch.arange(s["table"].shape[1] * page, device=DEV)
    cache, ids = s["cache"], s["table"].long()
    held = lambda x, sc: _values(x[ids], None if sc is None else sc[ids]).transpose(1, 2).reshape(B, Hkv, -1, d)         # noqa: E731
    z = q @ held(cache["k"], cache["k_scale"]).transpose(-1, -2)
    e = entry.view(1, 1, -1) - lens.view(B, 1, 1)                                        # < 0: before the new tokens
    mine = sees.gather(2, e.clamp(0, w - 1).expand(B, w, -1)) > 0
    seen = ((e < 0) & (sees.sum(-1, keepdim=True) > 0)) | ((e >= 0) & (e < w) & mine)     # [B,w,entries]
    seen = seen.repeat_interleave(G, 1).unsqueeze(1)
    z = z.masked_fill(~seen, -math.inf)
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, torch.zeros_like(m), m))
    del z
    sums = p.sum(-1, keepdim=True)
    out = (p @ held(cache["v"], cache["v_scale"])) / torch.where(sums == 0, torch.ones_like(sums), sums)
    out = out.view(B, Hkv, w, G, d).permute(0, 2, 1, 3, 4).reshape(B, w, Hq, d).to(BF16)
    lse = (m + torch.log(sums)).view(B, Hkv, w, G).permute(0, 1, 3, 2).reshape(B, Hq, w)
    return {"out": out, "lse": lse}


def _plain_logprob(s):
    c, x = s["case"], s["logits"].to(F32)
    N, V = c["N"], c["V"]
    m = x.amax(-1, keepdim=True)
    log_z = m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))
    logp = x - log_z
    r = {"logprob": logp.gather(1, s["tokens"].long().unsqueeze(-1)).squeeze(-1), "entropy": -(torch.exp(logp) * logp).sum(-1)}
    if c["top"]:
        bits = (x + 0.0).view(I32).to(torch.int64)                                       # order of numbers as order of integers; ties: the lowest place
        key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * 2 ** 20 + (2 ** 20 - 1 - torch.arange(V, device=DEV))
        r["top_id"] = (2 ** 20 - 1 - key.topk(c["top"], -1).values % 2 ** 20).to(I32)
        r["top_logprob"] = logp.gather(1, r["top_id"].long())
    if c["group"]:
        r["nll"] = -r["logprob"].view(-1, c["group"]).sum(-1)
    return r


def _plain(s):
    kind = s["case"]["kind"]
    return _plain_append(s) if kind == "append" else _plain_tree(s) if kind == "tree" else _plain_logprob(s)


# ------------------------------------------------------------------------------------ the framework's calls
def _framework(s):
    import paper_2502_14317_b200 as pc
    c = s["case"]
    if c["kind"] == "logprob":
        r = pc.token_logprobs(s["logits"], s["tokens"], top=c["top"], group=c["group"], want_entropy=True)
        return {k: r[k] for k in ("logprob", "entropy") + (("top_id", "top_logprob") if c["top"] else ()) + (("nll",) if c["group"] else ())}
    cache = s["cache"]
    if c["kind"] == "tree":
        r = pc.tree_attn(s["q"], cache, s["table"], s["lens"], parents=s["parents"], rope_theta=c["theta"], max_len=c["n"], want_lse=True, buffers=s["keep"])
        return {"out": r["out"], "lse": r["lse"]}
    pc.page_append(cache, s["k"], s["v"], s["table"], at=s["lens"], rope_theta=c["theta"], pos0=c["far"], parents=s["parents"], pick=s["pick"],
                   count=s["count"])
    if c["fmt"] == "bf16":
        return {"k": cache["k"], "v": cache["v"]}
    k, v = pc.kv_dequantize(cache)
    return {"k": k, "v": v, "k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_quantised(x, fmt):
    """values and scales of the rows of x, from the definition: the code is the number of the format nearest to x / a * Q"""
    a = x.abs().amax(-1, keepdim=True)
    y = torch.where(a >= TINY, x / a * TOP[fmt], torch.zeros_like(x))
    if fmt == "int8":
        code = torch.round(y)
    else:
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3.0)       # 3 bits behind the first; subnormals
        code = torch.round(y / step) * step
    scale = torch.where(a >= TINY, a / TOP[fmt], torch.zeros_like(a))
    return code * scale, scale.squeeze(-1)


def _paths(parents, w, B):
    """for each sequence and token the list of tokens that it sees, by walking up; [] where it is not there"""
    if parents is None:
        return [[list(range(i + 1)) for i in range(w)] for _ in range(B)]
    paths = []
    for row in parents.tolist():
        mine = []
        for i, p in enumerate(row):
            mine.append([] if p < -1 else [i] if p == -1 else mine[p] + [i])
        paths.append(mine)
    return paths


def _turned(x, pos, theta):
    """rows x [n,H,d] at positions [n], by complex numbers"""
    d = x.shape[-1]
    angle = torch.outer(torch.as_tensor(pos, device=DEV, dtype=F64), torch.as_tensor([theta ** (-2.0 * t / d) for t in range(d // 2)], device=DEV, dtype=F64))
    z = torch.complex(x[..., :d // 2].to(F64), x[..., d // 2:].to(F64)) * torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "logprob":
        r = {k: torch.empty(c["N"], device=DEV, dtype=F64) for k in ("logprob", "entropy")}
        if c["top"]:
            r["top_id"], r["top_logprob"] = None, torch.empty((c["N"], c["top"]), device=DEV, dtype=F64)
        for i in range(c["N"]):
            logp = torch.log_softmax(s["logits"][i].to(F64), -1)
            r["logprob"][i] = logp[s["tokens"][i].long()]
            r["entropy"][i] = torch.special.entr(torch.exp(logp)).sum()
            if c["top"]:
                r["top_logprob"][i] = logp.topk(c["top"]).values
        if c["group"]:
            r["nll"] = torch.stack([-x.sum() for x in r["logprob"].split(c["group"])])
        return r
    B, Hkv, d, page, lens = c["B"], c["Hkv"], c["d"], c["page"], _lens(c)
    cache, table = s["cache"], s["table"].tolist()
    if c["kind"] == "append":
        r = {x: torch.zeros(cache[x].shape, device=DEV, dtype=F64) for x in ("k", "v")}
        if c["fmt"] != "bf16":
            r["k_scale"], r["v_scale"] = (torch.zeros(cache["k"].shape[:3], device=DEV, dtype=F64) for _ in range(2))
        for b in range(B):
            k, v, n, step = s["k"][b], s["v"][b], c["n"], list(range(c["n"]))
            if c["how"] == "accept":
                n = int(s["count"][b])
                k, v = k[s["pick"][b, :n].long()], v[s["pick"][b, :n].long()]
            if c["how"] == "tree":
                step = [len(p) - 1 for p in _paths(s["parents"][b:b + 1], c["n"], 1)[0] if p]       # (those that are not there are the last)
                n = len(step)
                k, v = k[:n], v[:n]
            if n == 0:
                continue
            k, v = _turned(k, [lens[b] + c["far"] + x for x in step[:n]], c["theta"]), v.to(F64)
            for x, rows in (("k", k), ("v", v)):
                if c["fmt"] != "bf16":
                    rows, scale = _exact_quantised(rows, c["fmt"])
                for first in range(lens[b] // page * page, lens[b] + n, page):                  # page by page
                    lo, hi = max(first, lens[b]), min(first + page, lens[b] + n)
                    r[x][table[b][first // page], :, lo - first:hi - first] = rows[lo - lens[b]:hi - lens[b]].transpose(0, 1)
                    if c["fmt"] != "bf16":
                        r[x + "_scale"][table[b][first // page], :, lo - first:hi - first] = scale[lo - lens[b]:hi - lens[b]].transpose(0, 1)
        return r
    w, Hq = c["w"], c["Hq"]
    G = Hq // Hkv
    if 4.0 * w * Hq * d * (sum(lens) + B * w) > 3.0e12:
        return None
    paths = _paths(s["parents"], w, B)
    out, lse = torch.zeros((B, w, Hq, d), device=DEV, dtype=F64), torch.full((B, Hq, w), -math.inf, device=DEV, dtype=F64)
    for b in range(B):
        n = lens[b] + w
        ids = s["table"][b, :-(-n // page)].long()
        depth = [max(len(p) - 1, 0) for p in paths[b]]
        q = _turned(s["q"][b], [lens[b] + x for x in depth], c["theta"]).to(BF16).to(F64)         # [w,Hq,d]
        hidden = torch.ones((w, n), dtype=torch.bool)
        for i, p in enumerate(paths[b]):
            if p:
                hidden[i, :lens[b]] = False
                hidden[i, [lens[b] + x for x in p]] = False
        hidden, there = hidden.to(DEV), torch.tensor([bool(p) for p in paths[b]], device=DEV)
        for h in range(Hkv):
            k, v = (cache[x][ids, h].to(F64) if cache[x + "_scale"] is None else cache[x][ids, h].to(F64) * cache[x + "_scale"][ids, h].to(F64).unsqueeze(-1)
                    for x in ("k", "v"))
            k, v = k.reshape(-1, d)[:n], v.reshape(-1, d)[:n]
            z = (torch.einsum("wgd,nd->gwn", q[:, h * G:(h + 1) * G], k) / math.sqrt(d)).masked_fill(hidden, -math.inf)
            o = torch.softmax(z, -1) @ v
            out[b, :, h * G:(h + 1) * G] = torch.where(there.view(1, w, 1), o, torch.zeros_like(o)).transpose(0, 1)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
    return {"out": out, "lse": lse}
