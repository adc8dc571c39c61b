"""The 8-bit caches and the attention over shared and own caches in 64 bits, on the CPU, from their definitions."""
import numpy as np
import torch

TOP = {"int8": 127.0, "e4m3": 448.0}


def quantise(x, fmt):
    """rows x [..., d] (bf16 values, float64) -> values the codes stand for and fp32 scales.

    The definition's three fp32 operations: r = Q / a, x * r, a / Q; the rounding to the format is done in 64 bits."""
    x = np.asarray(x, np.float64)
    a = np.abs(x).max(-1).astype(np.float32)
    finite, held = np.isfinite(a), np.isfinite(a) & (a >= np.float32(2.0 ** -100))
    top = np.float32(TOP[fmt])
    safe = np.where(held, a, np.float32(1))
    r, scale = (top / safe).astype(np.float32), (safe / top).astype(np.float32)
    with np.errstate(invalid="ignore"):
        y = (x.astype(np.float32) * r[..., None]).astype(np.float64)
        if fmt == "int8":
            code = np.rint(y)
        else:
            step = np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
            code = np.rint(y / step) * step
    code = np.where(held[..., None], code, 0.0)
    scale = np.where(held, scale, np.where(finite, np.float32(0), np.float32(np.nan)))
    return code, scale.astype(np.float32)


def to_bf16(x):
    """nearest bf16 of the float64 values x"""
    x = np.asarray(x, np.float64)
    f = x.astype(np.float32)
    toward = np.where(np.abs(f.astype(np.float64)) > np.abs(x), np.nextafter(f, np.float32(0)), f)     # towards zero ...
    bits = toward.view(np.uint32) | (toward.astype(np.float64) != x).astype(np.uint32)                 # ... and the rest as a sticky bit
    out = ((bits.astype(np.uint64) + 0x7FFF + ((bits >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(x), out, f)


def rotate(q, pos, theta):
    """q [B,w,H,d] float64 at positions pos [B,w] < 2^15 -> rotated in fp32 with fp32 angles, rounded to bf16.  The operations are torch's own
    on the GPU, whose pow, cos and sin of fp32 numbers are the ones that the definition means; test_rotation has it against 64 bits."""
    if theta == 0:
        return q
    d, f32 = q.shape[-1], torch.float32
    t = torch.arange(d // 2, device="cuda", dtype=f32)
    a = torch.tensor(pos, device="cuda", dtype=f32).unsqueeze(-1) * torch.pow(torch.tensor(theta, device="cuda", dtype=f32), -2.0 * t / d)
    c, s = torch.cos(a).unsqueeze(2), torch.sin(a).unsqueeze(2)
    x, y = torch.from_numpy(q).to("cuda", f32).split(d // 2, -1)
    return f64(torch.cat([x * c - y * s, y * c + x * s], -1).to(torch.bfloat16))


def attention(q, pos, theta, scale, prefix, n_prefix, own, lens, kw, vw):
    """q [B,w,Hq,d]; prefix, own: (k, v) values [B,Hkv,n,d] or None; lens [B]; kw, vw [B,w,Hkv,d] or None -> out, lse"""
    B, w, Hq, d = q.shape
    Hkv = (prefix or own or (kw.transpose(0, 2, 1, 3),))[0].shape[1]
    G = Hq // Hkv
    scale = scale or d ** -0.5
    q = rotate(q, pos, theta)
    out, lse = np.zeros((B, w, Hq, d)), np.full((B, Hq, w), -np.inf)
    for b in range(B):
        for h in range(Hkv):
            k, v = [], []
            if prefix is not None and n_prefix:
                k.append(prefix[0][0, h, :n_prefix]); v.append(prefix[1][0, h, :n_prefix])
            if own is not None:
                k.append(own[0][b, h, :lens[b]]); v.append(own[1][b, h, :lens[b]])
            n = sum(len(x) for x in k)
            if kw is not None:
                k.append(kw[b, :, h]); v.append(vw[b, :, h])
            k, v = np.concatenate(k), np.concatenate(v)
            for i in range(w):
                m = n + (i + 1 if kw is not None else 0)
                if m == 0:
                    continue
                for g in range(G):
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = k[:m] @ q[b, i, h * G + g] * scale
                        top = s.max()
                        e = np.exp(s - top)
                        out[b, i, h * G + g] = e @ v[:m] / e.sum()
                        lse[b, h * G + g, i] = top + np.log(e.sum())
    return out, lse


def f64(t):
    return t.detach().to(torch.float32).cpu().numpy().astype(np.float64)
