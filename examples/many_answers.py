"""Many answers to one long prompt, one attention layer: the prompt is compressed once and held in 8 bits, every answer has an
8-bit cache of its own, and all of them read the prompt's cache together.

    prompt          hot_path (chunks, ranking, eviction) -> gather_kv_quantize: the kept keys and values, 8 bits
    question        w new tokens per answer: cache_attn over the prompt (causal among themselves), kv_quantize into the own caches
    one token more  cache_attn over prompt, own cache and the token itself, kv_quantize behind the own cache; one CUDA graph

The layer's projections are random, so the answers mean nothing; the caches, positions and calls are those of a model's layer.
At the end the last step is computed again in plain PyTorch, over the caches read back with kv_dequantize.

    python examples/many_answers.py [--answers 16] [--steps 32] [--format int8|e4m3]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2502_14317_b200 as pc  # noqa: E402


def rotate(x, pos, theta):
    """rotate-half RoPE of x [B,n,H,d] at positions pos [B,n]"""
    d = x.shape[-1]
    angle = pos.float().unsqueeze(-1) * theta ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float32) / d)
    c, s = torch.cos(angle).unsqueeze(2), torch.sin(angle).unsqueeze(2)
    a, b = x.float().split(d // 2, -1)
    return torch.cat([a * c - b * s, b * c + a * s], -1).to(x.dtype)


class Layer:
    def __init__(self, Hq, Hkv, d, theta, seed):
        self.Hq, self.Hkv, self.d, self.theta = Hq, Hkv, d, theta
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda n, m: (torch.randn(n, m, generator=g, device="cuda") * n ** -0.5).to(torch.bfloat16)     # noqa: E731
        self.qkv, self.out = make(Hq * d, (Hq + 2 * Hkv) * d), make(Hq * d, Hq * d)

    def project(self, x):
        """x [B,n,Hq*d] -> q, k, v [B,n,H,d], unrotated"""
        y = (x @ self.qkv).view(*x.shape[:2], -1, self.d)
        return y[:, :, :self.Hq], y[:, :, self.Hq:self.Hq + self.Hkv], y[:, :, self.Hq + self.Hkv:]

    def tokens(self, attended):
        """the next tokens' states from what the layer attended to: its output, to unit size"""
        y = attended.flatten(2) @ self.out
        return (y / y.float().pow(2).mean(-1, keepdim=True).sqrt().clamp_min(1e-6).to(y.dtype)).to(torch.bfloat16)


def plain(q, k, v, kw, vw):
    """one new token, q [B,1,Hq,d] rotated, over k, v [B,Hkv,n,d] and itself, in fp32"""
    B, _, Hq, d = q.shape
    Hkv = k.shape[1]
    k, v = torch.cat([k, kw.transpose(1, 2)], 2).float(), torch.cat([v, vw.transpose(1, 2)], 2).float()
    s = torch.einsum("bhgd,bhnd->bhgn", q.view(B, Hkv, Hq // Hkv, d).float(), k) * d ** -0.5
    return torch.einsum("bhgn,bhnd->bhgd", s.softmax(-1), v).reshape(B, 1, Hq, d)


def run(answers=16, steps=32, fmt="int8", *, chunks=8, chunk_len=2048, question=12, Hq=32, Hkv=8, d=128, theta=5e5, m=4, k_keep=512, seed=0):
    torch.backends.cuda.matmul.allow_tf32 = False
    layer, g = Layer(Hq, Hkv, d, theta, seed), torch.Generator(device="cuda").manual_seed(seed + 1)
    noise = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)                  # noqa: E731

    # the prompt, once
    q, k, v = (t.contiguous() for t in layer.project(noise(chunks, chunk_len, Hq * d)))
    res = pc.hot_path(q, k, v, w=64, rope_theta=theta, m=m, k_keep=k_keep)
    prefix, _ = pc.gather_kv_quantize(res["k_rot"], v, res["kept"], res["idx"], format=fmt)
    del q, k, v

    # the question, another for every answer; the answers go on from the end of a chunk, where the path's query window stood
    own = pc.kv_cache(answers, Hkv, question + steps, d, fmt)
    pos = torch.full((answers,), chunk_len, dtype=torch.int32, device="cuda")
    lens = torch.zeros(answers, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q, kw, vw = layer.project(noise(answers, question, Hq * d))
    kw = rotate(kw, pos.unsqueeze(1) + torch.arange(question, device="cuda"), theta)
    got = pc.cache_attn(q, kw, vw, prefix=prefix, q_pos=pos, rope_theta=theta)
    assert got["status"].item() == 0
    pc.kv_quantize(own, kw, vw, at=lens, status=status)
    lens += question
    pos += question
    x = layer.tokens(got["out"])[:, -1:].contiguous()

    # token after token
    last, buffers = {}, {}

    def step():
        q, kw, vw = layer.project(x)
        kw = rotate(kw, pos.unsqueeze(1), theta)
        got = pc.cache_attn(q, kw, vw, prefix=prefix, own=own, own_len=lens, q_pos=pos, rope_theta=theta, buffers=buffers)
        pc.kv_quantize(own, kw, vw, at=lens, status=status)
        last.update(q=q, kw=kw, vw=vw, out=got["out"], status=got["status"], pos=pos.clone(), lens=lens.clone())
        x.copy_(layer.tokens(got["out"]))
        lens.add_(1)
        pos.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(steps - 1):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    assert last["status"].item() == 0 and status.item() == 0

    # the last step again
    n = int(last["lens"][0])
    pk, pv = pc.kv_dequantize(prefix)
    ok, ov = pc.kv_dequantize(own, n)
    keys, values = (torch.cat([a.expand(answers, -1, -1, -1), b], 2) for a, b in ((pk, ok), (pv, ov)))
    want = plain(rotate(last["q"], last["pos"].unsqueeze(1), theta), keys, values, last["kw"], last["vw"])
    off = ((last["out"].float() - want).abs().max() / want.abs().max()).item()
    bytes8 = sum(t.numel() * t.element_size() for c in (prefix, own) for t in (c["k"], c["v"], c["k_scale"], c["v_scale"]))
    bytes16 = sum(2 * t.numel() for c in (prefix, own) for t in (c["k"], c["v"]))
    return {"us_per_step": begin.elapsed_time(end) * 1e3 / max(steps - 1, 1), "relative_difference": off, "cache_bytes": bytes8, "bf16_cache_bytes": bytes16,
            "own_entries": int(lens[0])}


if __name__ == "__main__":
    args = argparse.ArgumentParser(description="Many answers over one compressed 8-bit prompt")
    args.add_argument("--answers", type=int, default=16)
    args.add_argument("--steps", type=int, default=32)
    args.add_argument("--format", choices=("int8", "e4m3"), default="int8")
    a = args.parse_args()
    r = run(a.answers, a.steps, a.format)
    print("%d answers, %d tokens each: %.1f us a step (projections included), caches %.1f MB (bf16: %.1f MB), last step off by %.1e of its largest value"
          % (a.answers, r["own_entries"], r["us_per_step"], r["cache_bytes"] / 1e6, r["bf16_cache_bytes"] / 1e6, r["relative_difference"]))
