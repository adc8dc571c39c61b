"""Paged caches, the attention of drafted tokens over them, and log probabilities in 64 bits, on the CPU, from their definitions."""
import numpy as np
import torch

from tests import cache_ref as ref


def turned(x, pos, theta):
    """rows x [..., H, d] float64 at positions pos [...]: pairs (t, t + d/2) by pos * theta^(-2t/d)"""
    if theta == 0:
        return x
    h = x.shape[-1] // 2
    a = np.asarray(pos, np.float64)[..., None] * theta ** (-np.arange(h) / h)
    c, s = np.cos(a)[..., None, :], np.sin(a)[..., None, :]
    u, v = x[..., :h], x[..., h:]
    return np.concatenate([u * c - v * s, v * c + u * s], -1)


def near_a_border(x, pos, theta):
    """Pairs [..., H, d/2] of which a rotated element lies so near the middle between two bf16 numbers that fp32 may round it to either.

    The rotation in fp32 is off by at most 2^-20 (|u| + |v|): the angle by 2^-25 of a turn (2^-22.3), sine and cosine by 2^-23, products and their
    sum by 2^-24 each.  Twice that."""
    h = x.shape[-1] // 2
    y = turned(x, pos, theta)
    off = np.tile(2.0 ** -19 * (np.abs(x[..., :h]) + np.abs(x[..., h:])), 2)
    either = ref.to_bf16(y - off) != ref.to_bf16(y + off)
    return either[..., :h] | either[..., h:]


def seen(parents):
    """tokens that each of w tokens sees, by walking up; [] where it is not there"""
    out = []
    for i, p in enumerate(parents):
        out.append([i] if p == -1 else out[p] + [i] if 0 <= p < i and out[p] else [])
    return out


def chain(w):
    return list(range(-1, w - 1))


def values(cache):
    """what a pool stands for, float64 [pages,Hkv,page,d]"""
    if cache["format"] == "bf16":
        return ref.f64(cache["k"]), ref.f64(cache["v"])
    return tuple(ref.f64(cache[n]) * ref.f64(cache[n + "_scale"])[..., None] for n in ("k", "v"))


def attention(q, held, table, lens, parents, pos, theta, scale=0.0):
    """q [B,w,Hq,d] float64; held: values(); table [B,n]; lens [B] (negative: no such sequence); parents [B][w]; pos [B] -> out, lse"""
    B, w, Hq, d = q.shape
    k, v = held
    Hkv, page = k.shape[1], k.shape[2]
    G, scale = Hq // Hkv, scale or d ** -0.5
    out, lse = np.zeros((B, w, Hq, d)), np.full((B, Hq, w), -np.inf)
    for b in range(B):
        if lens[b] < 0:
            continue
        ids = [int(table[b][e]) for e in range((lens[b] + w + page - 1) // page)]
        paths = seen(parents[b])
        for h in range(Hkv):
            kk, vv = (np.concatenate([x[i, h] for i in ids]) for x in (k, v))
            for i, path in enumerate(paths):
                if not path:
                    continue
                which = list(range(lens[b])) + [lens[b] + j for j in path]
                for g in range(h * G, h * G + G):
                    row = q[b, i, g]
                    if theta:
                        row = ref.to_bf16(turned(row[None], np.float64(pos[b] + len(path) - 1), theta)[0])
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = kk[which] @ row * scale
                        e = np.exp(s - s.max())
                        out[b, i, g] = e @ vv[which] / e.sum()
                        lse[b, g, i] = s.max() + np.log(e.sum())
    return out, lse


def logprobs(x, tokens, top, scale=1.0):
    """x [N,V] float64 -> logprob [N], entropy [N], top_id [N,top], top_logprob [N,top]; rows of nothing but -inf as the definition has them"""
    z = x * scale
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = z.max(-1, keepdims=True)
        lp = z - m - np.log(np.exp(z - m).sum(-1, keepdims=True))
        none = np.isneginf(m[:, 0])
        lp[none] = -np.inf
        p = np.exp(lp)
        entropy = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0 * p).sum(-1)
    entropy[none] = 0
    ids = np.stack([np.lexsort((np.arange(x.shape[1]), -row))[:top] for row in x]) if top else None
    got = np.where(tokens < 0, 0.0, np.where(tokens < x.shape[1], lp[np.arange(len(x)), np.clip(tokens, 0, x.shape[1] - 1)], np.nan))
    return got, entropy, ids, None if ids is None else np.take_along_axis(lp, ids, -1)


def pool(pc, seed, B, lens, w, Hkv, page, d, fmt, spoil=True, big=1.0):
    """Pages in no order with lens[b] + w entries of every sequence; everything else is what nothing may use: NaN and large codes.

    -> cache, table (int32, CUDA)"""
    g = torch.Generator().manual_seed(seed)
    n_table = max((max(lens) + w + page - 1) // page, 1)
    pages = B * n_table + 2
    k, v = ((torch.randn(pages, page, Hkv, d, generator=g) * s).to(torch.bfloat16) for s in (big, 1.0))
    table = torch.randperm(pages, generator=g)[:B * n_table].view(B, n_table).to(torch.int32)
    if fmt == "bf16":
        cache = {"format": "bf16", "k": k.transpose(1, 2).contiguous().cuda(), "v": v.transpose(1, 2).contiguous().cuda()}
    else:
        cache = pc.kv_cache(pages, Hkv, page, d, fmt)
        pc.kv_quantize(cache, k.cuda(), v.cuda())
    if spoil:
        used = torch.zeros(pages, page, dtype=torch.bool)
        for b in range(B):
            for e in range(max(lens[b] + w, 0)):
                used[table[b, e // page], e % page] = True
        stale = ~used.unsqueeze(1).expand(pages, Hkv, page).cuda()
        for name in ("k", "v"):
            if fmt == "bf16":
                cache[name][stale] = float("nan")
            else:
                cache[name].view(torch.uint8)[stale] = 0x7F
                cache[name + "_scale"][stale] = float("nan")
    return cache, table.cuda()
