"""Performance cases of the 8-bit key/value cache and of attention over caches that a batch may share.

Kinds of work (field ``kind``):
  write  ``kv_quantize``: n new tokens of B sequences go into their 8-bit caches, and what was written is read back
  evict  ``gather_kv_quantize``: the kept tokens of a compressed prompt go into an 8-bit cache, and are read back
  read   ``kv_dequantize``: entries of an 8-bit cache as bf16
  attn   ``cache_attn``: w new tokens of B sequences attend to a prefix that all of them share (``n_prefix`` entries), to their own
         caches (up to ``n_own`` entries, ``ragged``: of different lengths) and to themselves (causal)

Inputs follow the distributions that the repository's tests and benchmark draw: N(0,1) queries, keys and values and an attention
sink, with a few channels of the keys several times larger than the others, as keys have them.
"""
import math

import torch

own = False
DEV = "cuda"
BF16 = torch.bfloat16
F32 = torch.float32
TOP = {"int8": 127.0, "e4m3": 448.0}                     # largest code of a format
TINY = 2.0 ** -100                                       # rows below it are stored as zeros


def _write(name, B, n, Hkv, d, fmt, at, ragged=False, fused=False):
    """at: entries that are there before; ragged: a different number in each sequence; fused: keys and values are slices of one projection"""
    return {"name": name, "kind": "write", "B": B, "n": n, "Hkv": Hkv, "d": d, "fmt": fmt, "at": at, "ragged": ragged, "fused": fused}


def _evict(name, C, L, w, Hkv, d, m, k, fmt):
    return {"name": name, "kind": "evict", "C": C, "L": L, "w": w, "Hkv": Hkv, "d": d, "m": m, "k": k, "fmt": fmt}


def _read(name, B, n, Hkv, d, fmt):
    return {"name": name, "kind": "read", "B": B, "n": n, "Hkv": Hkv, "d": d, "fmt": fmt}


def _attn(name, B, w, Hq, Hkv, d, theta, n_prefix, prefix_fmt, n_own, own_fmt, ragged):
    return {"name": name, "kind": "attn", "B": B, "w": w, "Hq": Hq, "Hkv": Hkv, "d": d, "theta": theta, "n_prefix": n_prefix,
            "prefix_fmt": prefix_fmt, "n_own": n_own, "own_fmt": own_fmt, "ragged": ragged}


def listed():
    return [
        # the new token of one sequence: latency
        _write("write-token", 1, 1, 8, 128, "int8", 16384),
        # windows of 16 tokens of 64 sequences of different lengths, small heads, out of a fused projection
        _write("write-ragged-d64", 64, 16, 2, 64, "e4m3", 4000, ragged=True, fused=True),
        # a 128K prompt after eviction: 8 of 16 chunks, 2048 tokens of each per kv-head
        _evict("evict-128k", 16, 8192, 64, 8, 128, 8, 2048, "e4m3"),
        # a short cache back to bf16
        _read("read-b1-d64", 1, 1001, 2, 64, "int8"),
        # caches of a batch back to bf16, for a stage that takes bf16
        _read("read-b64", 64, 4096, 8, 128, "int8"),
        # one generation step of one sequence over its compressed cache: latency
        _attn("decode-b1", 1, 1, 32, 8, 128, 5.0e5, 0, "", 16401, "int8", False),
        # one generation step of 64 sequences, each with a compressed cache of its own: the memory's rate
        _attn("decode-b64", 64, 1, 32, 8, 128, 5.0e5, 0, "", 16384, "int8", False),
        # drafts of 4 tokens of 23 sequences of different lengths, small heads, 28 rows per kv-head
        _attn("draft-ragged-d64", 23, 4, 14, 2, 64, 1.0e6, 0, "", 5000, "e4m3", True),
        # the query window of one prompt over its compressed cache
        _attn("window-b1", 1, 64, 32, 8, 128, 5.0e5, 16384, "int8", 0, "", False),
        # a few answers to one short prompt, small heads
        _attn("answers-b5-d64", 5, 3, 4, 2, 64, 1.0e4, 777, "bf16", 40, "bf16", True),
        # 64 continuations of one compressed prompt
        _attn("shared-b64", 64, 1, 32, 8, 128, 5.0e5, 16384, "bf16", 512, "bf16", True),
        # 256 continuations of a long prompt, everything in 8 bits
        _attn("shared-b256", 256, 1, 32, 8, 128, 5.0e5, 65536, "e4m3", 200, "int8", True),
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))

    largest = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["write", "evict", "read", "attn", "attn", "shared", "shared"])
        d, fmt, Hkv = rng.choice([64, 128]), rng.choice(["int8", "e4m3"]), rng.choice([1, 2, 4, 8])
        if kind == "write":
            c = _write("", spread(1, 64), spread(1, 2048), Hkv, d, fmt, spread(1, 20000), rng.random() < 0.5, rng.random() < 0.5)
        elif kind == "evict":
            C, L, w = spread(1, 16), spread(200, 8192), spread(1, 64)
            c = _evict("", C, L, w, Hkv, d, rng.randint(1, C), spread(1, L - w), fmt)
        elif kind == "read":
            c = _read("", spread(1, 64), spread(1, 16384), Hkv, d, fmt)
        else:
            G = rng.choice([1, 2, 3, 4, 7, 8])
            theta = rng.choice([1.0e4, 5.0e5])
            formats = ["int8", "e4m3", "bf16"]
            if kind == "attn":
                B, w = spread(1, 64), spread(1, max(1, 32 // G))
                c = _attn("", B, w, G * Hkv, Hkv, d, theta, 0, "", spread(1, 20000), rng.choice(formats), rng.random() < 0.5)
            else:
                B = spread(1, 256)
                w = spread(1, 64) if B == 1 else spread(1, 8)
                n_own = 0 if rng.random() < 0.2 else spread(1, 1000)
                c = _attn("", B, w, G * Hkv, Hkv, d, theta, spread(100, 65536), rng.choice(formats), n_own,
                          rng.choice(formats) if n_own else "", n_own > 0 and rng.random() < 0.7)
        del c["name"]
        if _cost(c) <= largest:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.4e15)


def _row(fmt, d):
    """bytes of an entry of one head, keys or values"""
    return 2 * d if fmt == "bf16" else d + 4


def work(case):
    c = case
    Hkv, d = c["Hkv"], c["d"]
    if c["kind"] == "attn":
        lens = _lens(c)
        rows, G = c["B"] * c["w"] * c["Hq"], c["Hq"] // Hkv
        keys = sum(c["n_prefix"] + n for n in lens)
        pairs = c["Hq"] * (c["w"] * keys + c["B"] * c["w"] * (c["w"] + 1) // 2)
        cache = Hkv * 2 * (c["n_prefix"] * _row(c["prefix_fmt"], d) + sum(lens) * _row(c["own_fmt"], d))
        return {"bytes": cache + 4 * rows * d + 4 * (rows // G) * d + 4 * rows, "flops": 4 * pairs * d}
    entries = 2 * Hkv * (c["m"] * c["k"] if c["kind"] == "evict" else c["B"] * c["n"])
    q = _row(c["fmt"], d)
    # read: codes and scales in, bf16 out; else bf16 in, codes and scales out, and those read back
    return {"bytes": entries * (q + 2 * d if c["kind"] == "read" else 2 * d + q + q + 2 * d), "flops": 0}


def _lens(c):
    """valid entries of the sequences' own caches"""
    if not c["ragged"]:
        return [c["n_own"]] * c["B"]
    return [(c["n_own"] * ((37 * b + 11) % 101)) // 100 for b in range(c["B"])]


# ------------------------------------------------------------------------------------ inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=F32)


def _keys(gen, *shape):
    """keys [..., d]: N(0,1) with every 16th channel four times as large"""
    k = _normal(gen, *shape)
    k[..., ::16] *= 4.0
    return k.to(BF16)


def _codes(x, fmt):
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
    """what an 8-bit (or bf16) cache stands for, fp32"""
    return codes.to(F32) if scale is None else codes.to(F32) * scale.unsqueeze(-1)


def _fill(gen, B, Hkv, n, d, fmt):
    """a cache [B,Hkv,n,d] as a program has it: k, v and, in 8 bits, their scales"""
    k, v = torch.empty((2, B, Hkv, n, d), device=DEV, dtype=BF16 if fmt == "bf16" else torch.int8 if fmt == "int8" else torch.float8_e4m3fn)
    ks, vs = (None, None) if fmt == "bf16" else torch.empty((2, B, Hkv, n), device=DEV, dtype=F32)
    for b in range(B):
        x, y = _keys(gen, Hkv, n, d), _normal(gen, Hkv, n, d).to(BF16)
        x[:, :1] *= 4.0                                  # the sink
        if fmt == "bf16":
            k[b], v[b] = x, y
        else:
            k[b], ks[b] = _codes(x, fmt)
            v[b], vs[b] = _codes(y, fmt)
    return {"format": fmt, "k": k, "v": v, "k_scale": ks, "v_scale": vs}


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 17)
    Hkv, d, s = c["Hkv"], c["d"], {"case": c}
    if c["kind"] == "write":
        B, n = c["B"], c["n"]
        if c["fused"]:
            both = _keys(gen, B, n, 6 * Hkv, d)
            s["k"], s["v"] = both[:, :, 4 * Hkv:5 * Hkv], both[:, :, 5 * Hkv:]
        else:
            s["k"], s["v"] = _keys(gen, B, n, Hkv, d), _normal(gen, B, n, Hkv, d).to(BF16)
        s["at"] = c["at"]
        if c["ragged"]:
            s["at"] = torch.randint(0, c["at"] + 1, (B,), generator=gen, device=DEV, dtype=torch.int32)
        cap = c["at"] + n + 7
        kind = torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn
        s["cache"] = {"format": c["fmt"], "k": torch.zeros((B, Hkv, cap, d), device=DEV, dtype=torch.int8).view(kind),
                      "v": torch.zeros((B, Hkv, cap, d), device=DEV, dtype=torch.int8).view(kind),
                      "k_scale": torch.zeros((B, Hkv, cap), device=DEV), "v_scale": torch.zeros((B, Hkv, cap), device=DEV)}
    elif c["kind"] == "evict":
        C, L, m, k = c["C"], c["L"], c["m"], c["k"]
        s["k"], s["v"] = _keys(gen, C, L, Hkv, d), _normal(gen, C, L, Hkv, d).to(BF16)
        s["kept"] = torch.randperm(C, generator=gen, device=DEV)[:m].sort().values.to(torch.int32)
        score = torch.rand((m, Hkv, L - c["w"]), generator=gen, device=DEV)
        s["idx"] = score.topk(k, dim=-1).indices.sort(-1).values.to(torch.int32).contiguous()
        kind = torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn
        s["cache"] = {"format": c["fmt"], "k": torch.zeros((1, Hkv, m * k, d), device=DEV, dtype=torch.int8).view(kind),
                      "v": torch.zeros((1, Hkv, m * k, d), device=DEV, dtype=torch.int8).view(kind),
                      "k_scale": torch.zeros((1, Hkv, m * k), device=DEV), "v_scale": torch.zeros((1, Hkv, m * k), device=DEV)}
    elif c["kind"] == "read":
        s["cache"] = _fill(gen, c["B"], Hkv, c["n"], d, c["fmt"])
    else:
        B, w, Hq = c["B"], c["w"], c["Hq"]
        s["q"], s["kw"], s["vw"] = _normal(gen, B, w, Hq, d).to(BF16), _keys(gen, B, w, Hkv, d), _normal(gen, B, w, Hkv, d).to(BF16)
        s["prefix"] = _fill(gen, 1, Hkv, c["n_prefix"], d, c["prefix_fmt"]) if c["n_prefix"] else None
        s["own"] = _fill(gen, B, Hkv, c["n_own"], d, c["own_fmt"]) if c["n_own"] else None
        s["lens"] = torch.tensor(_lens(c), device=DEV, dtype=torch.int32)
        s["pos0"] = 4000                                 # position of the first new token behind an empty own cache
        s["keep"] = {}                                   # outputs and workspaces, kept from call to call
    return s


# ------------------------------------------------------------------------------------ plain form
def _rotate(q, pos0, pos, theta):
    """q [B,w,H,d] turned by its position (pairs (t, t + d/2)), rounded to bf16 as the definition has it"""
    B, w, _, d = q.shape
    t = torch.arange(d // 2, device=DEV, dtype=F32)
    p = (pos0 + pos).to(F32).view(B, 1) + torch.arange(w, device=DEV, dtype=F32)
    a = p.unsqueeze(-1) * torch.pow(torch.tensor(theta, device=DEV, dtype=F32), -2.0 * t / d)
    co, si = torch.cos(a).unsqueeze(2), torch.sin(a).unsqueeze(2)
    x, y = q[..., :d // 2].to(F32), q[..., d // 2:].to(F32)
    return torch.cat([x * co - y * si, y * co + x * si], -1).to(BF16).to(F32)


def _plain_attn(s):
    c = s["case"]
    B, w, Hq, Hkv, d = c["B"], c["w"], c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    q = _rotate(s["q"], s["pos0"], s["lens"], c["theta"]) / math.sqrt(d)
    q = q.view(B, w, Hkv, G, d).permute(2, 0, 1, 3, 4)                                   # [Hkv,B,w,G,d]
    causal = torch.arange(w, device=DEV).view(1, w) > torch.arange(w, device=DEV).view(w, 1)
    kw, vw = s["kw"].to(F32).permute(2, 0, 1, 3), s["vw"].to(F32).permute(2, 0, 1, 3)    # [Hkv,B,w,d]
    sw = (q.reshape(Hkv, B, w * G, d) @ kw.transpose(-1, -2)).view(Hkv, B, w, G, w)
    parts = [sw.masked_fill(causal.view(1, 1, w, 1, w), -math.inf).reshape(Hkv, B, w * G, w)]
    if s["prefix"] is not None:
        p = s["prefix"]
        kp, vp = _values(p["k"], p["k_scale"])[0], _values(p["v"], p["v_scale"])[0]
        parts.append((q.reshape(Hkv, B * w * G, d) @ kp.transpose(-1, -2)).view(Hkv, B, w * G, -1))
    if s["own"] is not None:
        o = s["own"]
        ko, vo = _values(o["k"], o["k_scale"]).transpose(0, 1), _values(o["v"], o["v_scale"]).transpose(0, 1)
        hidden = torch.arange(c["n_own"], device=DEV) >= s["lens"].view(1, B, 1, 1)
        parts.append((q.reshape(Hkv, B, w * G, d) @ ko.transpose(-1, -2)).masked_fill(hidden, -math.inf))
    m = parts[0].amax(-1, keepdim=True)
    m = torch.stack([m] + [x.amax(-1, keepdim=True) for x in parts[1:]]).amax(0)
    e = [torch.exp(x - m) for x in parts]
    l = torch.stack([x.sum(-1, keepdim=True) for x in e]).sum(0)
    out = e[0] @ vw
    if s["prefix"] is not None:
        out = out + (e[1].reshape(Hkv, B * w * G, -1) @ vp).view(Hkv, B, w * G, d)
    if s["own"] is not None:
        out = out + e[-1] @ vo
    out = (out / l).view(Hkv, B, w, G, d).permute(1, 2, 0, 3, 4).reshape(B, w, Hq, d).to(BF16)
    lse = (m + torch.log(l)).view(Hkv, B, w, G).permute(1, 0, 3, 2).reshape(B, Hq, w)
    return {"out": out, "lse": lse}


def _plain(s):
    c = s["case"]
    if c["kind"] == "attn":
        return _plain_attn(s)
    if c["kind"] == "read":
        p = s["cache"]
        return {"k": _values(p["k"], p["k_scale"]).to(BF16), "v": _values(p["v"], p["v_scale"]).to(BF16)}
    if c["kind"] == "write":
        k, v = s["k"].transpose(1, 2), s["v"].transpose(1, 2)
    else:
        m, k_keep, Hkv = c["m"], c["k"], c["Hkv"]
        chunk, head = s["kept"].long().view(m, 1, 1), torch.arange(Hkv, device=DEV).view(1, Hkv, 1)
        pick = lambda x: x[chunk, s["idx"].long(), head].transpose(0, 1).reshape(1, Hkv, m * k_keep, -1)  # noqa: E731
        k, v = pick(s["k"]), pick(s["v"])
    (kc, ks), (vc, vs) = _codes(k, c["fmt"]), _codes(v, c["fmt"])
    r = {"k": _values(kc, ks).to(BF16), "v": _values(vc, vs).to(BF16)}
    if c["kind"] == "evict" or not c["ragged"]:
        r.update(k_scale=ks, v_scale=vs)
    return r


# ------------------------------------------------------------------------------------ the framework's calls
def _framework(s):
    import paper_2502_14317_b200 as pc
    c = s["case"]
    if c["kind"] == "attn":
        r = pc.cache_attn(s["q"], s["kw"], s["vw"], prefix=s["prefix"], n_prefix=c["n_prefix"], own=s["own"], n_own=c["n_own"],
                          own_len=s["lens"] if c["ragged"] else None, q_pos0=s["pos0"] + (0 if c["ragged"] else c["n_own"]),
                          q_pos=s["lens"] if c["ragged"] else None, rope_theta=c["theta"], want_lse=True, buffers=s["keep"])
        return {"out": r["out"], "lse": r["lse"]}
    cache = s["cache"]
    if c["kind"] == "read":
        k, v = pc.kv_dequantize(cache, n=c["n"])
        return {"k": k, "v": v}
    if c["kind"] == "write":
        pc.kv_quantize(cache, s["k"], s["v"], at=s["at"])
        k, v = pc.kv_dequantize(cache, n=c["n"], at=s["at"])
        if c["ragged"]:
            return {"k": k, "v": v}
        a, e = c["at"], c["at"] + c["n"]
        return {"k": k, "v": v, "k_scale": cache["k_scale"][:, :, a:e], "v_scale": cache["v_scale"][:, :, a:e]}
    pc.gather_kv_quantize(s["k"], s["v"], s["kept"], s["idx"], cache)
    k, v = pc.kv_dequantize(cache, n=c["m"] * c["k"])
    return {"k": k, "v": v, "k_scale": cache["k_scale"], "v_scale": cache["v_scale"]}


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------------------------ in 64 bits
F64 = torch.float64


def _exact_quantised(x, fmt):
    """values and scales of the rows of x, from the definition: the code is the number of the format nearest to x / a * Q"""
    x = x.to(F64)
    a = x.abs().amax(-1, keepdim=True)
    y = torch.where(a >= TINY, x / a * TOP[fmt], torch.zeros_like(x))
    if fmt == "int8":
        code = torch.round(y)
    else:
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3.0)       # 3 bits behind the first; subnormals
        code = torch.round(y / step) * step
    scale = torch.where(a >= TINY, a / TOP[fmt], torch.zeros_like(a))
    return code * scale, scale.squeeze(-1)


def exact(case, seed):
    s, c = prepare(case, seed), case
    Hkv, d = c["Hkv"], c["d"]
    stored = lambda t, sc, b, h: t[b, h].to(F64) if sc is None else t[b, h].to(F64) * sc[b, h].to(F64).unsqueeze(-1)  # noqa: E731
    if c["kind"] == "read":
        p, r = s["cache"], {}
        for name in ("k", "v"):
            r[name] = torch.empty(p[name].shape, device=DEV, dtype=F64)
            for b in range(c["B"]):
                for h in range(Hkv):
                    r[name][b, h] = stored(p[name], p[name + "_scale"], b, h)
        return r
    if c["kind"] in ("write", "evict"):
        r = {}
        for name in ("k", "v"):
            x = s[name].transpose(1, 2)
            if c["kind"] == "evict":
                rows = [torch.cat([x[int(j), h][s["idx"][i, h].long()] for i, j in enumerate(s["kept"])]) for h in range(Hkv)]
                x = torch.stack(rows).unsqueeze(0)
            r[name], scale = _exact_quantised(x, c["fmt"])
            if c["kind"] == "evict" or not c["ragged"]:
                r[name + "_scale"] = scale
        return r
    B, w, Hq = c["B"], c["w"], c["Hq"]
    G, lens = Hq // Hkv, _lens(c)
    if B * w * Hq * (c["n_prefix"] + c["n_own"] + w) * d > 2.0e12:
        return None
    freq = float(c["theta"]) ** (-2.0 * torch.arange(d // 2, device=DEV, dtype=F64) / d)
    out, lse = torch.empty((B, w, Hq, d), device=DEV, dtype=F64), torch.empty((B, Hq, w), device=DEV, dtype=F64)
    visible = torch.ones((w, w), device=DEV, dtype=torch.bool).tril().repeat_interleave(G, 0)
    for h in range(Hkv):
        kp = vp = torch.empty((0, d), device=DEV, dtype=F64)
        if s["prefix"] is not None:
            kp, vp = (stored(s["prefix"][n], s["prefix"][n + "_scale"], 0, h) for n in ("k", "v"))
        for b in range(B):
            pos = s["pos0"] + lens[b] + torch.arange(w, device=DEV, dtype=F64)
            a = torch.outer(pos, freq).unsqueeze(1)
            x, y = s["q"][b, :, h * G:(h + 1) * G].to(F64).split(d // 2, -1)
            q = torch.cat([x * a.cos() - y * a.sin(), x * a.sin() + y * a.cos()], -1).to(BF16).to(F64).reshape(w * G, d)
            k, v = [kp, s["kw"][b, :, h].to(F64)], [vp, s["vw"][b, :, h].to(F64)]
            if lens[b]:
                k.insert(1, stored(s["own"]["k"], s["own"]["k_scale"], b, h)[:lens[b]])
                v.insert(1, stored(s["own"]["v"], s["own"]["v_scale"], b, h)[:lens[b]])
            k, v = torch.cat(k), torch.cat(v)
            z = q @ k.T / math.sqrt(d)
            z[:, -w:] = torch.where(visible, z[:, -w:], torch.full_like(z[:, -w:], -math.inf))
            out[b, :, h * G:(h + 1) * G] = (torch.softmax(z, -1) @ v).view(w, G, d)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, -1).view(w, G).T
    return {"out": out, "lse": lse}
