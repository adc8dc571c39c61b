"""New keys and values into paged caches against 64 bits, through the public call."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import cache_ref as ref
from tests import tree_ref as tree

pytestmark = pytest.mark.gpu
FORMATS = ["bf16", "int8", "e4m3"]


def _normal(seed, *shape, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pool(fmt, B, Hkv, page, d, most):
    n_table = (most + page - 1) // page
    pages = B * n_table + 2
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(5))[:B * n_table].view(B, n_table).to(torch.int32).cuda()
    cache = pc.kv_cache(pages, Hkv, page, d, fmt)
    for name in ("k", "v"):
        cache[name].view(torch.uint8).fill_(0x5A)
        if fmt != "bf16":
            cache[name + "_scale"].fill_(7.0)
    return cache, table


def _bytes(cache, name):
    return cache[name].contiguous().view(torch.uint8).cpu().numpy()


def _compare(cache, before, table, fmt, written, theta):
    """written: {(sequence, entry): (key [Hkv,d], value [Hkv,d], position)}, float64; every other byte of the pool is as it was"""
    page, d = cache["k"].shape[2:]
    tab = table.cpu().numpy()
    untouched = np.ones(cache["k"].shape[:3], bool)
    held = {n: ref.f64(cache[n]) for n in ("k", "v")}
    scales = {n: ref.f64(cache[n + "_scale"]) for n in ("k", "v")} if fmt != "bf16" else None
    for (b, e), (k, v, pos) in written.items():
        p, i = int(tab[b, e // page]), e % page
        untouched[p, :, i] = False
        want = tree.turned(k, pos, theta)
        if fmt == "bf16":
            assert np.array_equal(held["v"][p, :, i], v)
            # rounded once; where fp32 may round either way, one of the two: a step is at most 2^-7 of the value
            exact = ref.to_bf16(want).astype(np.float64)
            either = np.tile(tree.near_a_border(k, pos, theta), 2) if theta else np.zeros(want.shape, bool)
            assert np.array_equal(held["k"][p, :, i][~either], exact[~either])
            assert (np.abs(held["k"][p, :, i] - want) <= 2.0 ** -7 * np.abs(want) + 1e-30)[either].all()
            continue
        code, scale = ref.quantise(v, fmt)
        assert np.array_equal(held["v"][p, :, i], code) and np.array_equal(scales["v"][p, :, i], scale)
        if theta == 0:
            code, scale = ref.quantise(k, fmt)
            assert np.array_equal(held["k"][p, :, i], code) and np.array_equal(scales["k"][p, :, i], scale)
            continue
        a = np.abs(want).max(-1, keepdims=True)
        top = ref.TOP[fmt]
        got = held["k"][p, :, i] * scales["k"][p, :, i][:, None]
        # the largest magnitude is off by 2^-20 (|u| + |v|) <= 2^-19.5 of itself (see near_a_border), so the scale is; half a step of the format, and what the rotation is off
        assert (np.abs(scales["k"][p, :, i] - a[:, 0] / top) <= 2.0 ** -19 * a[:, 0] / top).all()
        step = a / top * 0.5 if fmt == "int8" else np.maximum(np.abs(want) * 2.0 ** -4, a / top * 2.0 ** -10)
        assert (np.abs(got - want) <= step * (1 + 2.0 ** -10) + 2.0 ** -17 * a).all()
    mask = torch.from_numpy(untouched)
    for name in ("k", "v") + (() if fmt == "bf16" else ("k_scale", "v_scale")):
        x, y = _bytes(cache, name), before[name]
        width = x.shape[-1] // (d if name in ("k", "v") else page)
        x, y = (t.reshape(*untouched.shape, -1) for t in (x, y))
        assert np.array_equal(x[mask.numpy()], y[mask.numpy()]), (name, width)


def _snapshot(cache):
    return {n: _bytes(cache, n).copy() for n in ("k", "v", "k_scale", "v_scale") if cache.get(n) is not None}


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("theta", [0.0, 5.0e5])
@pytest.mark.parametrize("B,n,Hkv,d,page,at", [(1, 1, 1, 64, 16, 0), (1, 1, 8, 128, 64, 63), (3, 1, 2, 64, 16, 15), (2, 17, 3, 128, 16, 9), (1, 100, 5, 64, 48, 31),
                                               (2, 257, 4, 128, 128, 100), (1, 1000, 2, 64, 32, 1)])
def test_rows_and_what_lies_beside_them(fmt, theta, B, n, Hkv, d, page, at):
    cache, table = _pool(fmt, B, Hkv, page, d, at + n)
    before = _snapshot(cache)
    k, v = _normal(1, B, n, Hkv, d), _normal(2, B, n, Hkv, d)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pc.page_append(cache, k.cuda(), v.cuda(), table, at=at, rope_theta=theta, status=status)
    kk, vv = ref.f64(k), ref.f64(v)
    _compare(cache, before, table, fmt, {(b, at + j): (kk[b, j], vv[b, j], at + j) for b in range(B) for j in range(n)}, theta)
    assert status.item() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_counts_and_sequences_that_are_not_there(fmt, d):
    """Slices of one projection, a start per sequence, fewer tokens of some, padding; positions that are not the entries'; far positions."""
    B, n, Hkv, page, theta = 6, 9, 2, 16, 1e4
    at, count, pos = [0, 31, -1, 17, 35, 5], [9, 3, 9, 0, 100, -4], [7, 100000, 3, 2 ** 30, 0, 9]
    cache, table = _pool(fmt, B, Hkv, page, d, 48)
    before = _snapshot(cache)
    both = _normal(3, B, n, 7 * Hkv, d).cuda()
    k, v = both[:, :, Hkv:2 * Hkv], both[:, :, 3 * Hkv:4 * Hkv]
    pc.page_append(cache, k, v, table, at=_i32(at), count=_i32(count), pos=_i32(pos), pos0=11, rope_theta=theta)
    kk, vv = ref.f64(k), ref.f64(v)
    written = {(b, at[b] + j): (kk[b, j], vv[b, j], 11 + pos[b] + j) for b in range(B) if at[b] >= 0 for j in range(min(max(count[b], 0), n))}
    assert len(written) == 9 + 3 + 9
    _compare(cache, before, table, fmt, written, theta)


@pytest.mark.parametrize("fmt", FORMATS)
def test_accepted_tokens(fmt):
    """pick: tokens of a longer source, the same twice, none; a table whose rows lie apart, a picking with a stride."""
    B, m, n_src, Hkv, d, page, theta = 3, 5, 12, 2, 128, 32, 5e5
    at = [30, 0, 61]
    pick = [[0, 2, 3, 7, 11], [4, 4, -1, 12, 5], [1, 2 ** 31 - 1, -2 ** 31, 0, 2]]
    cache, table = _pool(fmt, B, Hkv, page, d, 96)
    before = _snapshot(cache)
    wide = torch.full((B, 8), -3, dtype=torch.int32, device="cuda")
    wide[:, 1:4], wide_pick = table, _i32([[9] + x + [9] for x in pick])
    k, v = _normal(4, B, n_src, Hkv, d).cuda(), _normal(5, B, n_src, Hkv, d).cuda()
    pc.page_append(cache, k, v, wide[:, 1:4], at=_i32(at), pick=wide_pick[:, 1:6], count=_i32([5, 5, 4]), rope_theta=theta)
    kk, vv = ref.f64(k), ref.f64(v)
    written = {(b, at[b] + j): (kk[b, s], vv[b, s], at[b] + j) for b in range(B) for j, s in enumerate(pick[b]) if 0 <= s < n_src and j < (5, 5, 4)[b]}
    _compare(cache, before, table, fmt, written, theta)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [1, 6, 33, 64])
def test_drafted_tokens_stand_in_order_and_turn_by_depth(fmt, n):
    B, Hkv, d, page, theta = 2, 3, 64, 16, 1e4
    g = np.random.default_rng(n)
    parents = [[int(g.integers(max(-1, i - 4), i)) for i in range(n)] for _ in range(B)]
    parents[1] = [x if i != n // 2 else -2 for i, x in enumerate(parents[1])]
    at = [13, 40]
    cache, table = _pool(fmt, B, Hkv, page, d, 104)
    before = _snapshot(cache)
    k, v = _normal(6, B, n, Hkv, d), _normal(7, B, n, Hkv, d)
    pc.page_append(cache, k.cuda(), v.cuda(), table, at=_i32(at), parents=_i32(parents), rope_theta=theta, pos0=1000)
    kk, vv = ref.f64(k), ref.f64(v)
    written = {(b, at[b] + j): (kk[b, j], vv[b, j], 1000 + at[b] + len(p) - 1) for b in range(B) for j, p in enumerate(tree.seen(parents[b])) if p}
    _compare(cache, before, table, fmt, written, theta)


@pytest.mark.parametrize("fmt", FORMATS)
def test_entries_that_have_no_page(fmt):
    """Beyond the table, and pages that are none: not written, reported; the rest is."""
    cache, table = _pool(fmt, 2, 2, 16, 64, 40)
    table = table.clone()
    before = _snapshot(cache)
    bad = table.clone()
    bad[0, 1], bad[1, 0] = -1, cache["k"].shape[0]
    k, v, status = _normal(8, 2, 30, 2, 64), _normal(9, 2, 30, 2, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    pc.page_append(cache, k.cuda(), v.cuda(), bad, at=_i32([10, 25]), status=status)
    kk, vv = ref.f64(k), ref.f64(v)
    written = {(b, e): (kk[b, e - a], vv[b, e - a], 0) for b, a in ((0, 10), (1, 25)) for e in range(a, min(a + 30, 48)) if not (b == 0 and 16 <= e < 32)}
    _compare(cache, before, table, fmt, written, 0.0)
    assert status.item() == 421


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_rows_that_are_not_finite_read_back_as_nan(fmt):
    x = _normal(10, 1, 5, 1, 64)
    x[0, 1, 0, 7], x[0, 2, 0, 9] = float("nan"), float("inf")
    cache = pc.kv_cache(1, 1, 8, 64, fmt)
    pc.page_append(cache, x.cuda(), x.cuda(), _i32([[0]]), at=2, rope_theta=1e4)
    for got in pc.kv_dequantize(cache):
        got = ref.f64(got)[0, 0]
        assert np.isnan(got[3:5]).all() and np.isfinite(got[[0, 1, 2, 5, 6, 7]]).all()


def test_a_pool_beyond_2_31_elements():
    Hkv, d, page = 8, 128, 256
    pages = 2 ** 31 // (Hkv * page * d) + 3
    cache = {"format": "bf16", "k": torch.zeros(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda"),
             "v": torch.zeros(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda")}
    k, v = _normal(11, 1, 20, Hkv, d).cuda(), _normal(12, 1, 20, Hkv, d).cuda()
    pc.page_append(cache, k, v, _i32([[0, pages - 1]]), at=page)
    assert torch.equal(cache["k"][-1, :, :20], k[0].transpose(0, 1)) and torch.equal(cache["v"][-1, :, :20], v[0].transpose(0, 1))
    assert not cache["k"][:-1].any() and not cache["v"][:-1].any() and not cache["k"][-1, :, 20:].any()


def test_a_captured_call():
    cache, table = _pool("bf16", 2, 2, 16, 64, 64)
    k, v, at = _normal(13, 2, 3, 2, 64).cuda(), _normal(14, 2, 3, 2, 64).cuda(), _i32([5, 30])
    other = dict(cache, k=cache["k"].clone(), v=cache["v"].clone())
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        pc.page_append(cache, k, v, table, at=at, rope_theta=1e4)
        at += 3
    for _ in range(2):
        graph.replay()
    assert at.tolist() == [11, 36]
    for start in ([5, 30], [8, 33]):
        pc.page_append(other, k, v, table, at=_i32(start), rope_theta=1e4)
    assert torch.equal(cache["k"].view(torch.int16), other["k"].view(torch.int16)) and torch.equal(cache["v"].view(torch.int16), other["v"].view(torch.int16))


def test_refusals():
    cache, table = pc.kv_cache(6, 2, 16, 64, "int8"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    k = torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    good = dict(cache=cache, k=k, v=k, table=table, at=44)
    pc.page_append(cache, k, k, table, at=44)
    for change in (dict(at=45), dict(at=-1), dict(at=None), dict(at=_i32([1])), dict(k=k.float()), dict(v=k[:, :3]), dict(k=k[..., :32], v=k[..., :32]), dict(k=k[:, :, :1], v=k[:, :, :1]),
                   dict(table=table.long()), dict(table=table[:1]), dict(table=None), dict(count=_i32([1])), dict(pos=_i32([1])), dict(pick=_i32([[1]])),
                   dict(pick=_i32([[1], [1]]), parents=_i32([[1], [1]])), dict(parents=_i32([[0, 1], [0, 1]])), dict(rope_theta=-1.0), dict(rope_theta=float("inf")),
                   dict(status=torch.zeros(1, device="cuda")), dict(pos0=2 ** 40), dict(cache=pc.kv_cache(6, 2, 20, 64, "int8")), dict(cache=dict(cache, v=None)),
                   dict(k=k.cpu(), v=k.cpu()), dict(k=torch.zeros(2, 65, 2, 64, dtype=torch.bfloat16, device="cuda"), v=torch.zeros(2, 65, 2, 64, dtype=torch.bfloat16, device="cuda"),
                                                    table=table.repeat(1, 4), at=0, parents=torch.full((2, 65), -1, dtype=torch.int32, device="cuda"))):
        a = dict(good, **change)
        with pytest.raises(pc.PcError):
            pc.page_append(a.pop("cache"), a.pop("k"), a.pop("v"), a.pop("table"), **a)
