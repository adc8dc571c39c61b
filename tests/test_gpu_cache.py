"""8-bit caches and the attention over shared and own caches against 64 bits, through the public calls."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import cache_ref as ref

pytestmark = pytest.mark.gpu
FORMATS = ["int8", "e4m3"]
NAN = float("nan")


def _normal(seed, *shape, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def _ints(t):
    return t.view(torch.uint8).cpu().numpy() if t.dtype is torch.float8_e4m3fn else t.cpu().numpy()


def _values(cache):
    """what a cache stands for, float64 [B,Hkv,capacity,d]"""
    if cache["format"] == "bf16":
        return ref.f64(cache["k"]), ref.f64(cache["v"])
    return tuple(ref.f64(cache[n]) * ref.f64(cache[n + "_scale"])[..., None] for n in ("k", "v"))


def _rows(seed, B, n, Hkv, d):
    """ordinary rows, zeros, rows near and below the smallest that are held, very large ones, ties"""
    x = _normal(seed, B, n, Hkv, d)
    flat = x.view(-1, d)
    for i in range(flat.shape[0]):
        case = i % 11
        if case == 3:
            flat[i] = 0
        elif case == 5:
            flat[i] *= 2.0 ** -99
        elif case == 6:
            flat[i] = flat[i].clamp(-0.9, 0.9) * 2.0 ** -101
        elif case == 7:
            flat[i] *= 2.0 ** 120
        elif case == 8:
            flat[i] = torch.arange(d) - d // 2 + 0.5                  # halves of a step where a / Q = 1
            flat[i, 0] = 127.0
        elif case == 9:
            flat[i, 1:] = 0
    return x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,B,n,Hkv", [(128, 1, 1, 1), (64, 1, 1, 1), (128, 3, 37, 2), (64, 5, 100, 3), (128, 2, 1000, 8), (64, 1, 3001, 1)])
def test_quantised_rows(fmt, d, B, n, Hkv):
    """Codes and scales as the definition gives them, to the bit; what is read back is code * scale rounded once."""
    k, v = _rows(1, B, n, Hkv, d), _rows(2, B, n, Hkv, d)
    at = 5
    cache = pc.kv_cache(B, Hkv, at + n + 3, d, fmt)
    pc.kv_quantize(cache, k.cuda(), v.cuda(), at=at)
    for x, name in ((k, "k"), (v, "v")):
        code, scale = ref.quantise(ref.f64(x).transpose(0, 2, 1, 3), fmt)
        got, got_scale = ref.f64(cache[name]), cache[name + "_scale"].cpu().numpy()
        assert np.array_equal(got[:, :, at:at + n], code)
        assert np.array_equal(got_scale[:, :, at:at + n], scale)
        assert not got[:, :, :at].any() and not got[:, :, at + n:].any() and not got_scale[:, :, :at].any() and not got_scale[:, :, at + n:].any()
    kd, vd = pc.kv_dequantize(cache, n=n + 2, at=at)
    for got, full in zip((kd, vd), _values(cache)):
        assert np.array_equal(ref.f64(got), ref.to_bf16(full[:, :, at:at + n + 2]).astype(np.float64))


@pytest.mark.parametrize("fmt", FORMATS)
def test_rows_that_are_not_finite_read_back_as_nan(fmt):
    d = 128
    x = _normal(3, 1, 6, 1, d)
    x[0, 1, 0, 7], x[0, 2, 0, 9], x[0, 3, 0, 127] = NAN, float("inf"), -float("inf")
    cache = pc.kv_cache(1, 1, 6, d, fmt)
    pc.kv_quantize(cache, x.cuda(), x.cuda())
    got = ref.f64(pc.kv_dequantize(cache)[0])[0, 0]
    assert np.isnan(got[1:4]).all() and np.isfinite(got[[0, 4, 5]]).all()
    assert not _ints(cache["k"])[0, 0, 1:4].any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_strided_sources_and_different_lengths(fmt, d):
    """Slices of a fused projection, a broadcast head, one start per sequence; entries behind the capacity are left out and reported."""
    B, n, Hkv, cap = 4, 9, 2, 40
    both = _normal(4, B, n, 7 * Hkv, d).cuda()
    k, v = both[:, :, Hkv:2 * Hkv], both[:, :, 3 * Hkv:4 * Hkv]
    at = torch.tensor([0, 31, 17, 35], dtype=torch.int32, device="cuda")
    cache, status = pc.kv_cache(B, Hkv, cap, d, fmt), torch.zeros(1, dtype=torch.int32, device="cuda")
    pc.kv_quantize(cache, k, v, at=at, status=status)
    assert status.item() == 401
    kd, vd = pc.kv_dequantize(cache, n=n, at=at)
    for b in range(B):
        there = min(n, cap - int(at[b]))
        for x, got, name in ((k, kd, "k"), (v, vd, "v")):
            code, scale = ref.quantise(ref.f64(x[b, :there]).transpose(1, 0, 2), fmt)
            assert np.array_equal(ref.f64(got[b])[:, :there], ref.to_bf16(code * scale[..., None].astype(np.float64)))
            assert not ref.f64(got[b])[:, there:].any()
            assert np.count_nonzero(cache[name + "_scale"][b].cpu().numpy()) == there * Hkv
    head = _normal(5, B, n, 1, d).cuda().expand(B, n, Hkv, d)
    pc.kv_quantize(cache, head, head, at=3)
    got = ref.f64(pc.kv_dequantize(cache, n=n, at=3)[0])
    assert np.array_equal(got[:, 0], got[:, 1]) and got.any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("C,L,Hkv,d,m,k", [(4, 64, 2, 64, 2, 17), (3, 200, 1, 128, 3, 1), (5, 129, 8, 128, 2, 100)])
def test_gather_into_an_8_bit_cache(fmt, C, L, Hkv, d, m, k):
    """What gather_kv followed by kv_quantize gives, positions -1 as zeros."""
    ks, vs = _normal(6, C, L, Hkv, d).cuda(), _normal(7, C, L, Hkv, d).cuda()
    gen = torch.Generator().manual_seed(8)
    kept = torch.randperm(C, generator=gen)[:m].sort().values.to(torch.int32).cuda()
    idx = torch.stack([torch.randperm(L, generator=gen)[:k].sort().values for _ in range(m * Hkv)]).view(m, Hkv, k).to(torch.int32)
    if k > 2:
        idx[0, 0, -2:] = -1
    idx = idx.cuda()
    cache, pos = pc.gather_kv_quantize(ks, vs, kept, idx, format=fmt, want_pos=True)
    kc, vc, want_pos = pc.gather_kv(ks, vs, kept, idx)
    other = pc.kv_cache(1, Hkv, m * k, d, fmt)
    pc.kv_quantize(other, kc.transpose(0, 1).unsqueeze(0), vc.transpose(0, 1).unsqueeze(0))
    assert torch.equal(pos, want_pos)
    for n in ("k", "v"):
        assert np.array_equal(_ints(cache[n]), _ints(other[n])) and torch.equal(cache[n + "_scale"], other[n + "_scale"])


# ------------------------------------------------------------------------------------ attention
def _cache(seed, B, Hkv, n, extra, d, fmt, scale=1.0):
    """n valid entries, then `extra` that nothing may use: NaN and large codes"""
    k, v = _normal(seed, B, n + extra, Hkv, d, scale=scale), _normal(seed + 1, B, n + extra, Hkv, d)
    if fmt == "bf16":
        cache = {"format": "bf16", "k": k.transpose(1, 2).contiguous().cuda(), "v": v.transpose(1, 2).contiguous().cuda()}
    else:
        cache = pc.kv_cache(B, Hkv, n + extra, d, fmt)
        pc.kv_quantize(cache, k.cuda(), v.cuda())
    _spoil(cache, [n] * B)
    return cache


def _spoil(cache, lens):
    for b, n in enumerate(lens):
        for name in ("k", "v"):
            if cache["format"] == "bf16":
                cache[name][b, :, n:] = NAN
            else:
                cache[name].view(torch.uint8)[b, :, n:] = 0x7F            # NaN of e4m3
                cache[name + "_scale"][b, :, n:] = NAN


def _check(got, want, what, lse, want_lse):
    """Outputs are bf16 (half a step: 2^-9 of the value) of sums whose weights were rounded to bf16 in the widest case (2^-9 of
    sum p |v| <= max |v|, some 4.5 here; many keys average it away, one key has it whole) -> |error| <= 2^-8 |ref| + 2^-9 * 4.5 = 9e-3.
    lse: fp32 exponentials and sums, and logits in fp32 (|q| |k| up to some 60 * 2^-22 after scaling): 1e-4."""
    d = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (d <= 9e-3 + 2.0 ** -8 * np.abs(want)).all(), (what, d.max())
    assert np.sqrt((d ** 2).mean()) <= 3e-3 * max(1e-30, np.sqrt((want ** 2).mean())) + 1e-6, (what, np.sqrt((d ** 2).mean()))
    assert (np.abs(lse - want_lse) <= 1e-4 + 1e-5 * np.abs(want_lse)).all(), (what, np.abs(lse - want_lse).max())


def _run(B, w, Hq, Hkv, d, n_prefix, pf, n_own, of, *, ragged=False, window=True, theta=1.0e4, seed=20, scale=0.0, extra=9, big=1.0):
    q = _normal(seed, B, w, Hq, d)
    kw, vw = (_normal(seed + 1, B, w, Hkv, d), _normal(seed + 2, B, w, Hkv, d)) if window else (None, None)
    prefix = _cache(seed + 3, 1, Hkv, n_prefix, extra, d, pf, big) if n_prefix else None
    own = _cache(seed + 5, B, Hkv, n_own, extra, d, of, big) if n_own else None
    lens = [n_own] * B
    kwargs = {}
    if ragged:
        lens = [(n_own * ((7 * b + 3) % 11)) // 10 for b in range(B)]
        _spoil(own, lens)
        kwargs = {"own_len": torch.tensor(lens, dtype=torch.int32, device="cuda"), "q_pos": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    got = pc.cache_attn(q.cuda(), *(None if x is None else x.cuda() for x in (kw, vw)), prefix=prefix, n_prefix=n_prefix, own=own, n_own=n_own,
                        q_pos0=300, rope_theta=theta, softmax_scale=scale, want_lse=True, **kwargs)
    assert got["status"].item() == 0
    pos = 300 + np.arange(w)[None] + (np.array(lens)[:, None] if ragged else np.zeros((B, 1)))
    clean = lambda c: None if c is None else tuple(np.nan_to_num(x) for x in _values(c))       # noqa: E731
    want, want_lse = ref.attention(ref.f64(q), pos, theta, scale, clean(prefix), n_prefix, clean(own), lens,
                                   *(None if x is None else ref.f64(x) for x in (kw, vw)))
    _check(ref.f64(got["out"]), want, "out", got["lse"].cpu().numpy().astype(np.float64), want_lse)
    return got


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n", [
    (1, 1, 1, 1, 64, 1), (1, 1, 1, 1, 128, 1), (1, 1, 8, 2, 128, 15), (2, 1, 8, 2, 128, 16), (2, 1, 8, 2, 64, 17), (1, 2, 7, 1, 128, 63),
    (1, 1, 4, 4, 64, 64), (3, 1, 8, 1, 128, 65), (2, 5, 6, 2, 64, 127), (1, 3, 10, 2, 128, 129), (1, 4, 8, 1, 128, 1000), (2, 8, 8, 2, 64, 777),
    (1, 1, 32, 8, 128, 5000), (1, 33, 2, 2, 64, 300), (2, 17, 4, 1, 128, 400), (1, 128, 1, 1, 64, 130)])
def test_attention_over_own_caches(fmt, B, w, Hq, Hkv, d, n):
    _run(B, w, Hq, Hkv, d, 0, "", n, fmt)


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("window", [True, False])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n", [(11, 1, 8, 2, 128, 100), (11, 3, 4, 1, 64, 257), (12, 4, 14, 2, 64, 130)])
def test_sequences_of_different_lengths(fmt, window, B, w, Hq, Hkv, d, n):
    """Lengths from zero on; with nothing to see at all a row is zeros and its lse -infinity."""
    got = _run(B, w, Hq, Hkv, d, 0, "", n, fmt, ragged=True) if window else None
    if window:
        return
    lens = torch.tensor([0, n] + [1] * (B - 2), dtype=torch.int32, device="cuda")
    cache = _cache(40, B, Hkv, n, 3, d, fmt)
    _spoil(cache, lens.tolist())
    q = _normal(41, B, w, Hq, d)
    got = pc.cache_attn(q.cuda(), own=cache, n_own=n, own_len=lens, want_lse=True)
    assert not ref.f64(got["out"][0]).any() and (got["lse"][0] == -float("inf")).all() and got["status"].item() == 0
    want, want_lse = ref.attention(ref.f64(q), None, 0, 0, None, 0, tuple(np.nan_to_num(x) for x in _values(cache)), lens.tolist(), None, None)
    _check(ref.f64(got["out"][1:]), want[1:], "out", got["lse"][1:].cpu().numpy(), want_lse[1:])


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("ragged", [True, False])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n", [(3, 40, 4, 2, 64, 300), (11, 24, 4, 1, 128, 400), (2, 70, 8, 2, 128, 1000), (5, 33, 2, 1, 128, 129), (12, 20, 8, 2, 64, 2500),
                                            (1, 128, 4, 1, 128, 5000), (1, 128, 8, 2, 64, 1), (13, 9, 16, 2, 128, 128)])
def test_many_rows_over_own_caches(fmt, ragged, B, w, Hq, Hkv, d, n):
    """More than 32 rows of a kv-head in every sequence; lengths from zero on, NaN codes behind them."""
    _run(B, w, Hq, Hkv, d, 0, "", n, fmt, ragged=ragged)


@pytest.mark.parametrize("pf,of", [("int8", "e4m3"), ("bf16", "int8"), ("e4m3", "bf16")])
@pytest.mark.parametrize("window", [True, False])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n_prefix,n_own", [(3, 34, 4, 2, 128, 300, 200), (1, 12, 4, 1, 64, 20000, 700), (2, 64, 8, 2, 128, 129, 3000)])
def test_many_rows_over_prefix_and_own_caches(pf, of, window, B, w, Hq, Hkv, d, n_prefix, n_own):
    _run(B, w, Hq, Hkv, d, n_prefix, pf, n_own, of, ragged=True, window=window)


@pytest.mark.parametrize("pf,of", [("bf16", "bf16"), ("int8", "int8"), ("e4m3", "bf16"), ("bf16", "int8"), ("int8", "e4m3"), ("e4m3", "")])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n_prefix,n_own", [
    (2, 1, 4, 2, 64, 100, 7), (5, 1, 8, 2, 128, 700, 33), (3, 4, 8, 1, 128, 500, 64), (40, 1, 8, 2, 128, 300, 20), (9, 5, 14, 2, 64, 1030, 5),
    (3, 37, 4, 2, 128, 260, 1), (70, 2, 4, 1, 64, 129, 9), (150, 1, 8, 2, 128, 257, 3), (1, 64, 8, 2, 128, 900, 1), (2, 128, 4, 1, 128, 1, 1)])
def test_attention_over_a_shared_prefix(pf, of, B, w, Hq, Hkv, d, n_prefix, n_own):
    _run(B, w, Hq, Hkv, d, n_prefix, pf, n_own if of else 0, of, ragged=bool(of))


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("rows", [1, 20, 300])
def test_long_prefix_in_many_splits(fmt, rows):
    _run(rows, 1, 2, 2, 128, 20000, fmt, 0, "")


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("B", [2, 90])
def test_logits_that_grow_along_the_cache(fmt, B):
    """The reference maximum is raised again and again; scales of keys and values from 2^-20 to 2^20 beside one another."""
    Hq, Hkv, d, n = 4, 2, 128, 700
    q = _normal(50, B, 1, Hq, d)
    k, v = _normal(51, 1, n, Hkv, d), _normal(52, 1, n, Hkv, d)
    k = (k.float() * torch.linspace(0.01, 2.5, n).view(1, n, 1, 1)).to(torch.bfloat16)
    v = (v.float() * torch.exp2((torch.arange(n) * 37 % 41 - 20).float()).view(1, n, 1, 1)).to(torch.bfloat16)
    if fmt == "bf16":
        cache = {"format": "bf16", "k": k.transpose(1, 2).contiguous().cuda(), "v": v.transpose(1, 2).contiguous().cuda()}
    else:
        cache = pc.kv_cache(1, Hkv, n, d, fmt)
        pc.kv_quantize(cache, k.cuda(), v.cuda())
    got = pc.cache_attn(q.cuda(), prefix=cache, want_lse=True)
    vals = _values(cache)
    want, want_lse = ref.attention(ref.f64(q), None, 0, 0, vals, n, None, [0] * B, None, None)
    size, _ = ref.attention(ref.f64(q), None, 0, 0, (vals[0], np.abs(vals[1])), n, None, [0] * B, None, None)
    # weights rounded to bf16 (2^-9 each), values to bf16 where many rows share them (2^-9), the output once more
    assert (np.abs(ref.f64(got["out"]) - want) <= 1.01 * 2.0 ** -8 * size + 2.0 ** -8 * np.abs(want)).all()
    assert np.abs(got["lse"].cpu().numpy() - want_lse).max() <= 1e-4 + 1e-5 * np.abs(want_lse).max()


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("B", [1, 60])
def test_values_that_are_not_finite_reach_their_rows(fmt, B):
    """A NaN among the entries that count is not lost; an infinite logit neither."""
    k, v = _normal(60, 1, 200, 2, 64), _normal(61, 1, 200, 2, 64)
    v[0, 150, 1, 5] = NAN
    cache = {"format": "bf16", "k": k.transpose(1, 2).contiguous().cuda(), "v": v.transpose(1, 2).contiguous().cuda()}
    if fmt != "bf16":
        cache = pc.kv_cache(1, 2, 200, 64, fmt)
        pc.kv_quantize(cache, k.cuda(), v.cuda())
    out = ref.f64(pc.cache_attn(_normal(62, B, 1, 4, 64).cuda(), prefix=cache)["out"])
    assert np.isfinite(out[:, :, :2]).all() and np.isnan(out[:, :, 2:, 5]).all()


@pytest.mark.parametrize("d,theta", [(64, 1.0e4), (128, 5.0e5)])
@pytest.mark.parametrize("pos", [0, 1, 4095, 8191, 32766, 32767, 32768, 1000000, 2 ** 30])
def test_rotation(d, theta, pos):
    """The rotated queries themselves: sequence t sees a key that is the t-th unit vector (value 1) and a zero key, so that its lse is
    log(1 + exp(q_t)).  Below 2^15 the fp32 angle is off by at most 2^-22 of itself, above by nothing; fp32 products and sums take 2^-21.  q_t is the
    bf16 number nearest to something in that interval, and is read out of the lse, whose slope is sigmoid(q_t) >= 0.01, to 100 * 2^-20."""
    q = _normal(75, 1, 2, 1, d)
    k = torch.zeros(d, 1, 2, d, dtype=torch.bfloat16)
    k[torch.arange(d), 0, 0, torch.arange(d)] = 1.0
    cache = {"format": "bf16", "k": k.cuda(), "v": torch.zeros_like(k).cuda()}
    lse = pc.cache_attn(q.cuda().expand(d, 2, 1, d), own=cache, q_pos0=5, q_pos=torch.full((d,), pos - 5, dtype=torch.int32, device="cuda"),
                        rope_theta=theta, softmax_scale=1.0, want_lse=True)["lse"].cpu().numpy().astype(np.float64)
    got = np.log(np.expm1(lse))[:, 0].T                                   # [w, d]
    x, y = ref.f64(q)[0, :, 0, :d // 2], ref.f64(q)[0, :, 0, d // 2:]
    a = (pos + np.arange(2))[:, None] * float(theta) ** (-2.0 * np.arange(d // 2) / d)
    want = np.concatenate([x * np.cos(a) - y * np.sin(a), y * np.cos(a) + x * np.sin(a)], -1)
    size = np.hypot(x, y)
    size = np.concatenate([size, size], -1)
    off = np.where(pos + np.arange(2) < 2 ** 15, 2.0 ** -22, 0.0)[:, None] * np.concatenate([a, a], -1)
    low, high = (ref.to_bf16(want + sign * size * (off + 2.0 ** -21)) for sign in (-1, 1))
    assert (got >= low - 100 * 2.0 ** -20).all() and (got <= high + 100 * 2.0 ** -20).all()


def test_queries_of_any_size():
    """Queries become halves times a power of two of their row: very large and very small rows keep their bits."""
    for up in (2.0 ** -60, 1.0, 2.0 ** 30):
        q, k, v = _normal(70, 1, 1, 8, 128), _normal(71, 1, 300, 2, 128), _normal(72, 1, 300, 2, 128)
        cache = pc.kv_cache(1, 2, 300, 128, "int8")
        pc.kv_quantize(cache, k.cuda(), v.cuda())
        got = pc.cache_attn((q.float() * up).to(torch.bfloat16).cuda(), prefix=cache, softmax_scale=0.1 / up, want_lse=True)
        want, want_lse = ref.attention(ref.f64(q), None, 0, 0.1, _values(cache), 300, None, [0], None, None)
        _check(ref.f64(got["out"]), want, up, got["lse"].cpu().numpy(), want_lse)


def test_strided_queries_and_windows():
    B, w, Hq, Hkv, d = 3, 2, 4, 2, 128
    both = _normal(80, B, w, Hq + 2 * Hkv, d)
    q, kw, vw = both[:, :, :Hq], both[:, :, Hq:Hq + Hkv], both[:, :, Hq + Hkv:]
    dev = both.cuda()
    cache = _cache(81, B, Hkv, 100, 0, d, "int8")
    a = pc.cache_attn(dev[:, :, :Hq], dev[:, :, Hq:Hq + Hkv], dev[:, :, Hq + Hkv:], own=cache, q_pos0=9, rope_theta=5e5, want_lse=True)
    b = pc.cache_attn(q.contiguous().cuda(), kw.contiguous().cuda(), vw.contiguous().cuda(), own=cache, q_pos0=9, rope_theta=5e5, want_lse=True)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_same_results_every_time_on_any_stream_and_with_kept_buffers():
    q, kw, vw = _normal(90, 6, 2, 8, 128).cuda(), _normal(91, 6, 2, 2, 128).cuda(), _normal(92, 6, 2, 2, 128).cuda()
    prefix, own = _cache(93, 1, 2, 3000, 0, 128, "e4m3"), _cache(95, 6, 2, 50, 5, 128, "int8")
    call = lambda **kw_: pc.cache_attn(q, kw, vw, prefix=prefix, own=own, n_own=50, rope_theta=1e4, q_pos0=50, want_lse=True, **kw_)   # noqa: E731
    first, keep = call(), {}
    small = pc.cache_attn(q[:1], kw[:1], vw[:1], prefix=prefix, n_prefix=10, buffers=keep)
    assert small["out"].shape == (1, 2, 8, 128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            again = call(buffers=keep)
            assert torch.equal(again["out"], first["out"]) and torch.equal(again["lse"], first["lse"])
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("pf,of", [("int8", ""), ("e4m3", "int8"), ("bf16", "e4m3"), ("", "int8"), ("", "bf16")])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n_prefix,n_own", [(256, 1, 32, 8, 128, 9000, 100), (128, 1, 32, 8, 64, 9000, 30), (64, 1, 32, 8, 128, 5000, 700),
                                                         (70, 2, 8, 8, 128, 3000, 50), (20, 1, 16, 4, 64, 4000, 2000), (2, 40, 8, 2, 128, 5000, 90)])
def test_calls_in_a_row(pf, of, B, w, Hq, Hkv, d, n_prefix, n_own):
    """Calls that follow each other without a pause, on other inputs in between, give the bits of calls on an idle GPU."""
    if not pf:
        n_prefix = 0
    states = []
    for seed in (200, 220, 240):
        q, kw, vw = _normal(seed, B, w, Hq, d).cuda(), _normal(seed + 1, B, w, Hkv, d).cuda(), _normal(seed + 2, B, w, Hkv, d).cuda()
        prefix = _cache(seed + 3, 1, Hkv, n_prefix, 0, d, pf) if pf else None
        own = _cache(seed + 5, B, Hkv, n_own, 0, d, of) if of else None
        states.append((q, kw, vw, dict(prefix=prefix, own=own, rope_theta=1e4, q_pos0=100, want_lse=True, buffers={})))
    call = lambda s: pc.cache_attn(*s[:3], **s[3])                                    # noqa: E731
    alone = []
    for s in states:
        torch.cuda.synchronize()
        r = call(s)
        torch.cuda.synchronize()
        alone.append((r["out"].clone(), r["lse"].clone()))
    for i in range(12):
        for j in (1, 2, 0):
            r = call(states[(i + j) % 3])
        assert torch.equal(r["out"], alone[i % 3][0]) and torch.equal(r["lse"], alone[i % 3][1]), i
        assert r["status"].item() == 0


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_a_later_token_that_is_no_number_stays_where_it_is_seen(fmt):
    """Windows of more and of fewer than 8 tokens: NaN and infinity in a token's key or value reach no earlier row."""
    for w, B in ((40, 1), (12, 20), (5, 3)):
        q, kw, vw = _normal(150, B, w, 4, 64), _normal(151, B, w, 2, 64), _normal(152, B, w, 2, 64)
        cache = _cache(153, 1, 2, 300, 0, 64, fmt)
        want = ref.f64(pc.cache_attn(q.cuda(), kw.cuda(), vw.cuda(), prefix=cache)["out"])
        t = w - 3
        vw[:, t, 1, 5], kw[:, t + 1, 1, 9] = NAN, float("inf")
        got = ref.f64(pc.cache_attn(q.cuda(), kw.cuda(), vw.cuda(), prefix=cache)["out"])
        assert np.abs(got[:, :t] - want[:, :t]).max() <= 2.0 ** -7 * np.abs(want).max()      # a row's keys may be taken another way: a bf16 step
        assert np.abs(got[:, :, :2] - want[:, :, :2]).max() <= 2.0 ** -7 * np.abs(want).max()
        assert np.isnan(got[:, t:, 2:, 5]).all()


def test_broadcast_windows():
    """Keys and values of new tokens that are the same for all heads or sequences, through strides of 0, as copies of them give."""
    for w in (3, 20):
        q, one = _normal(160, 4, w, 4, 64).cuda(), _normal(161, 4, w, 1, 64).cuda()
        cache = _cache(162, 1, 2, 200, 0, 64, "int8")
        for win in (one.expand(4, w, 2, 64), one[:1].expand(4, w, 1, 64).repeat(1, 1, 2, 1)[:1].expand(4, w, 2, 64)):
            a = pc.cache_attn(q, win, win, prefix=cache, want_lse=True)
            b = pc.cache_attn(q, win.contiguous(), win.contiguous(), prefix=cache, want_lse=True)
            # w = 20: strides of 0 take the keys one by one, copies go through the matrix units: P in bf16 (2^-9), the output a step
            assert (a["out"].float() - b["out"].float()).abs().max() <= 2.0 ** -6 * b["out"].float().abs().max()
            assert (a["lse"] - b["lse"]).abs().max() <= 1e-4


def test_decoding_steps_over_a_growing_cache():
    """Step after step: attend, then append; the same as one call with the window over all of them."""
    B, Hq, Hkv, d, n0, steps = 2, 4, 2, 64, 30, 5
    prefix = _cache(100, 1, Hkv, 200, 0, d, "int8")
    own = pc.kv_cache(B, Hkv, n0 + steps, d, "int8")
    pc.kv_quantize(own, _normal(102, B, n0, Hkv, d).cuda(), _normal(103, B, n0, Hkv, d).cuda())
    lens = torch.full((B,), n0, dtype=torch.int32, device="cuda")
    for t in range(steps):
        q, kw, vw = _normal(110 + t, B, 1, Hq, d), _normal(120 + t, B, 1, Hkv, d), _normal(130 + t, B, 1, Hkv, d)
        got = pc.cache_attn(q.cuda(), kw.cuda(), vw.cuda(), prefix=prefix, own=own, n_own=n0 + steps, own_len=lens, q_pos=lens, rope_theta=1e4, want_lse=True)
        want, want_lse = ref.attention(ref.f64(q), np.full((B, 1), n0 + t), 1e4, 0, _values(prefix), 200, _values(own), [n0 + t] * B, ref.f64(kw), ref.f64(vw))
        _check(ref.f64(got["out"]), want, t, got["lse"].cpu().numpy(), want_lse)
        pc.kv_quantize(own, kw.cuda(), vw.cuda(), at=lens)
        lens += 1


@pytest.mark.parametrize("fmt,capacity", [("int8", 17_000_003), ("bf16", 9_000_001)])
@pytest.mark.parametrize("B", [1, 40])
def test_offsets_beyond_32_bits(fmt, capacity, B):
    """Two kv-heads of a cache whose second begins beyond 2^31 bytes (int8) and elements, read from end to end: zeros but for its last entries.
    A zero key has weight 1 and adds nothing, so the answer is a sum over the last ones."""
    Hkv, d, n = 2, 128, 60
    q = _normal(170, B, 1, Hkv, d)
    k, v = _normal(171, 1, n, Hkv, d), _normal(172, 1, n, Hkv, d)
    for j in range(min(B, n)):
        k[0, j] = (q[j, 0].float() * 1.5).to(torch.bfloat16)             # a logit of some 17: as much as the zeros together
    cache = pc.kv_cache(1, Hkv, capacity, d, fmt)
    if fmt == "bf16":
        cache["k"][:, :, -n:], cache["v"][:, :, -n:] = k.transpose(1, 2).cuda(), v.transpose(1, 2).cuda()
        ks, vs = ref.f64(k.transpose(1, 2)), ref.f64(v.transpose(1, 2))
    else:
        small = pc.kv_cache(1, Hkv, n, d, fmt)
        pc.kv_quantize(small, k.cuda(), v.cuda())
        pc.kv_quantize(cache, k.cuda(), v.cuda(), at=capacity - n)
        got = pc.kv_dequantize(cache, n, at=torch.tensor([capacity - n], dtype=torch.int32, device="cuda"))
        assert all(torch.equal(x, y) for x, y in zip(got, pc.kv_dequantize(small)))
        assert not cache["k"][:, :, :-n].any() and not cache["v_scale"][:, :, :-n].any()
        ks, vs = _values(small)
    got = pc.cache_attn(q.cuda(), prefix=cache, want_lse=True)
    assert got["status"].item() == 0
    e = np.exp(np.einsum("bhd,hnd->bhn", ref.f64(q[:, 0]), ks[0]) * d ** -0.5)
    total = e.sum(-1) + capacity - n
    _check(ref.f64(got["out"])[:, 0], np.einsum("bhn,hnd->bhd", e, vs[0]) / total[..., None], "out", got["lse"][..., 0].cpu().numpy(), np.log(total))


def test_a_wait_that_runs_out_is_reported():
    """Nothing is broken for it: the limit is set so low that an ordinary wait for a copy may exceed it; the call returns and the next is right."""
    lib = pc.load_library()
    cache, q = _cache(140, 1, 2, 9000, 0, 128, "int8"), _normal(142, 1, 1, 8, 128).cuda()
    want = pc.cache_attn(q, prefix=cache)["out"].clone()
    lib.pc_debug_bounded_wait_test(1, 0)
    try:
        status = pc.cache_attn(q, prefix=cache)["status"].item()
    finally:
        lib.pc_debug_bounded_wait_test(0, 0)
    assert status in (0, 411, 412)
    got = pc.cache_attn(q, prefix=cache)
    assert got["status"].item() == 0 and torch.equal(got["out"], want)


def test_refusals():
    q, kw = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    one, two = pc.kv_cache(1, 2, 16, 64, "int8"), pc.kv_cache(2, 2, 16, 64, "int8")
    for args, kwargs in [((q,), {}), ((q, kw), {}), ((q, kw, kw[:1]), {}), ((q.float(), kw, kw), {}), ((q, kw, kw), {"prefix": two}), ((q, kw, kw), {"own": one}),
                         ((q, kw, kw), {"prefix": one, "n_prefix": 17}), ((q, kw, kw), {"n_own": 3}), ((q, kw, kw), {"rope_theta": -1.0}),
                         ((q, kw, kw), {"q_pos0": -1}), ((q, kw, kw), {"own": two, "own_len": torch.zeros(2, device="cuda")}),
                         ((q, kw, kw), {"own": two, "own_len": torch.zeros(3, dtype=torch.int32, device="cuda")}),
                         ((q, kw, kw), {"out": torch.empty(2, 1, 4, 64, device="cuda")}), ((q[..., :32], kw, kw), {}),
                         ((q, kw, kw), {"prefix": dict(one, k_scale=None)}), ((q, kw, kw), {"prefix": dict(one, format="int4")})]:
        with pytest.raises(pc.PcError):
            pc.cache_attn(*args, **kwargs)
    for bad in (lambda: pc.kv_quantize(two, kw, kw, at=16), lambda: pc.kv_quantize(two, kw, kw, at=-1), lambda: pc.kv_quantize(one, kw, kw),
                lambda: pc.kv_quantize(two, kw, kw[:, :, :1]), lambda: pc.kv_quantize({"format": "bf16", "k": kw, "v": kw}, kw, kw),
                lambda: pc.kv_dequantize(two, n=0), lambda: pc.kv_cache(1, 1, 1, 64, "int4"), lambda: pc.kv_quantize(two, kw, kw.float())):
        with pytest.raises(pc.PcError):
            bad()
