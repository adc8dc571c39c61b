"""Attention of drafted tokens over paged caches at its edges, on both kernels: positions before the first, values that are no number, values of any size."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import cache_ref as ref
from tests import tree_ref as tree
from tests.tree_edges import SHAPES

pytestmark = pytest.mark.gpu
FORMATS = ["bf16", "int8", "e4m3"]
NAN, INF = float("nan"), float("inf")


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _room(table, page, most):
    """the table with room for `most` entries, by pages that are none, which no sequence comes to"""
    more = max((most + page - 1) // page - table.shape[1], 0)
    return torch.cat([table, torch.full((len(table), more), -7, dtype=torch.int32, device="cuda")], 1)


# size of every seventh entry's values and of the others', as powers of two; every `zeros`-th row is zeros
SIZES = [(0, 0, 2), (20, 20, 2), (28, 28, 3), (60, 60, 2), (60, -60, 3), (100, 100, 5), (100, 0, 3), (100, -95, 4), (0, -95, 5000), (-60, -60, 2), (-92, -92, 3),
         (-97, -97, 5000), (-99, -99, 2)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,w,Hq,most,kernel", SHAPES[1:4])
def test_sizes_of_values_weigh_nothing(fmt, d, B, w, Hq, most, kernel):
    """An entry's weight is its key's, however large or small its value is, zeros among them, and the output is right relative to its own size."""
    Hkv, page, n = 2, 64, 900
    g = torch.Generator().manual_seed(60)
    pages = (n + w + page - 1) // page
    k, x = (torch.randn(pages, page, Hkv, d, generator=g) for _ in range(2))
    q = _normal(61, 1, w, Hq, d)
    table = _room(torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages), page, most + w).expand(B, -1)
    k, at = (k * 0.7).to(torch.bfloat16).cuda(), torch.arange(pages * page).view(pages, page, 1, 1)
    for big, rest, zeros in SIZES:
        v = (x * torch.exp2(torch.where(at % 7 == 3, float(big), float(rest))) * (at % zeros != 1)).to(torch.bfloat16)
        cache = pc.kv_cache(pages, Hkv, page, d, fmt)
        pc.kv_quantize(cache, k, v.cuda())
        got = pc.tree_attn(q.cuda().expand(B, -1, -1, -1), cache, table, _i32([n] * B), max_len=most, want_lse=True)
        held = tree.values(cache)
        want, want_lse = tree.attention(ref.f64(q), held, table.cpu().numpy(), [n], [tree.chain(w)], [0], 0)
        size, _ = tree.attention(ref.f64(q), (held[0], np.abs(held[1])), table.cpu().numpy(), [n], [tree.chain(w)], [0], 0)
        # Weights rounded to bf16 or halves (2^-9 at most), the output to bf16 (2^-9): twice that.  What a half loses below 2^-14 of the largest product, 2^-25 of
        # 448 codes for 900 entries, is 2^-6 of a code, of sums of at least 100 that large ones have: 2^-12 of them.
        off, room = np.abs(ref.f64(got["out"]) - want), 1.01 * 2.0 ** -8 * size + 2.0 ** -8 * np.abs(want)
        assert (off <= room).all(), ((big, rest, zeros), np.nanmax(off / room))
        off = np.abs(got["lse"].cpu().numpy() - want_lse)
        assert (off <= 1e-4 + 1e-5 * np.abs(want_lse)).all(), ((big, rest, zeros), off.max())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,most,kernel", SHAPES[1:])
@pytest.mark.parametrize("n", [0, 100, 128, 1000])
def test_new_tokens_that_are_no_number_stay_where_they_are_seen(fmt, B, w, Hq, most, kernel, n):
    """Values and keys of drafted tokens that are no number: only the rows that see them have them, an infinity keeps its sign."""
    d, G = 128, Hq // 2
    lens = [max(n - b, 0) for b in range(B)]
    cache, table = tree.pool(pc, 54, B, lens, w, 2, 16, d, fmt)
    g = np.random.default_rng(55)
    parents = [[int(g.integers(max(-1, i - 4), i)) for i in range(w)] for _ in range(B)]
    q = _normal(56, B, w, Hq, d).cuda()
    call = lambda: pc.tree_attn(q, cache, _room(table, 16, most + w), _i32(lens), parents=_i32(parents), max_len=most, want_lse=True)       # noqa: E731
    clean, paths = call(), [tree.seen(p) for p in parents]
    was, lse = ref.f64(clean["out"]), clean["lse"].cpu().numpy()
    b, value, key = B - 1, min(w - 1, 2), w // 2
    at = lambda i: (int(table[b, (lens[b] + i) // 16]), (lens[b] + i) % 16)                             # noqa: E731
    (p0, e0), (p1, e1) = at(value), at(key)
    columns = list(range(d))
    if fmt == "bf16":
        cache["v"][p0, 1, e0, 7], cache["v"][p0, 1, e0, 8], cache["k"][p1, 0, e1, 3] = -INF, NAN, NAN
        columns = [7, 8]
    elif fmt == "int8":
        cache["v_scale"][p0, 1, e0], cache["k_scale"][p1, 0, e1] = NAN, NAN
    else:
        cache["v"].view(torch.uint8)[p0, 1, e0, 8], cache["k"].view(torch.uint8)[p1, 0, e1, 3] = 0xFF, 0x7F
        columns = [8]
    got = call()
    out, sees = ref.f64(got["out"]), [i for i in range(w) if value in paths[b][i]]
    if fmt == "bf16":
        assert np.isneginf(out[b][sees][:, G:, 7]).all()
    assert np.isnan(out[b][sees][:, G:][:, :, [8]]).all() and (len(columns) < d or np.isnan(out[b][sees][:, G:]).all())
    for i in sees:
        out[b][i, G:, columns] = was[b][i, G:, columns]
    for i in range(w):
        if key in paths[b][i]:
            assert np.isnan(out[b][i, :G]).all() and np.isnan(got["lse"][b, :G, i].cpu().numpy()).all()
            out[b][i, :G] = was[b][i, :G]
    assert np.array_equal(out, was)
    assert np.array_equal(got["lse"].cpu().numpy()[:, G:], lse[:, G:]) or np.abs(got["lse"].cpu().numpy() - lse)[:, G:].max() <= 264 * 2.0 ** -24 + 2.0 ** -18


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,page", [(64, 16), (128, 48), (128, 256)])
@pytest.mark.parametrize("B,w,Hq,most,kernel", SHAPES[2:])
def test_many_rows_over_short_sequences(fmt, d, page, B, w, Hq, most, kernel):
    """The kernel for many rows where pieces, tiles and pages end: no entries, a few, a tile and its neighbours; sequences and tokens that are not there."""
    lens = [0, 1, 127 - w, 128, 129, -1, 700, 1100][:B]
    cache, table = tree.pool(pc, 57, B, lens, w, 2, page, d, fmt)
    g = np.random.default_rng(58)
    parents = [[int(g.integers(max(-1, i - 4), i)) for i in range(w)] for _ in range(B)]
    parents[1] = [p if i < w // 3 else -2 for i, p in enumerate(parents[1])]
    q = _normal(59, B, w, Hq, d)
    got = pc.tree_attn(q.cuda(), cache, _room(table, page, most + w), _i32(lens), parents=_i32(parents), max_len=most, want_lse=True)
    assert got["status"].item() == 0
    want, want_lse = tree.attention(ref.f64(q), tuple(np.nan_to_num(x) for x in tree.values(cache)), table.cpu().numpy(), lens, parents, [0] * B, 0)
    there, lse, out = np.isfinite(want_lse), got["lse"].cpu().numpy(), ref.f64(got["out"])
    assert np.array_equal(there, np.isfinite(lse)) and (lse[~there] == -INF).all()
    # weights and, over codes, nothing else to bf16 or halves: 2 * 2^-9 of sum p |v| <= 4.5, the output half a step
    assert (np.abs(out - want) <= 1.8e-2 + 2.0 ** -8 * np.abs(want)).all()
    assert (np.abs(lse - want_lse)[there] <= 1e-4 + 1e-5 * np.abs(want_lse[there])).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,most,kernel", SHAPES)
def test_values_that_are_no_number_beside_the_new_tokens_reach_all(fmt, B, w, Hq, most, kernel):
    """A value of the context that is no number reaches every row, wherever it stands: of 200 entries the last eight share a unit of 16, and those from 128 on a tile,
    with the new tokens.  Weights do not depend on values: lse stays, and so does the other kv-head."""
    q, parents, G = _normal(53, B, w, Hq, 64).cuda(), _i32([-1] + [0] * (w - 1)), Hq // 2
    for n, spoiled in ((200, 89), (200, 150), (200, 191), (200, 192), (200, 199), (5, 0), (5, 4), (16, 15)):
        cache, table = tree.pool(pc, 52, B, [n] * B, w, 2, 16, 64, fmt)
        call = lambda c: pc.tree_attn(q, c, _room(table, 16, most + w), _i32([n] * B), parents=parents, max_len=most, want_lse=True)       # noqa: E731
        clean = call(cache)
        p, e, was = int(table[0, spoiled // 16]), spoiled % 16, ref.f64(clean["out"])
        for what in (NAN, INF) + (("code",) if fmt == "e4m3" else ()):
            spoil = {name: x.clone() if torch.is_tensor(x) else x for name, x in cache.items()}
            if what == "code":
                spoil["v"].view(torch.uint8)[p, 1, e, 5] = 0x7F
            elif fmt == "bf16":
                spoil["v"][p, 1, e] = what
            else:
                spoil["v_scale"][p, 1, e] = what
            got = call(spoil)
            out, hit = ref.f64(got["out"]), [5] if what == "code" else list(range(64))
            assert not np.isfinite(out[0][:, G:, hit]).any(), (n, spoiled, what)
            out[0][:, G:, hit] = was[0][:, G:, hit]
            assert np.array_equal(out, was) and torch.equal(got["lse"][1:], clean["lse"][1:]) and torch.equal(got["lse"][0, :G], clean["lse"][0, :G]), (n, spoiled, what)
            # sums of up to 264 positive terms in another order and with other roundings, 2^-24 each, of terms that fp32 exponents up to 2^5 make right to 2^-19
            assert (got["lse"] - clean["lse"]).abs().max() <= 264 * 2.0 ** -24 + 2.0 ** -18, (n, spoiled, what)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("w,Hq,first", [(1, 4, -1), (1, 4, -2), (4, 4, -4), (3, 14, -2), (20, 8, -9)])
def test_positions_before_the_first(fmt, d, w, Hq, first):
    """pos0 + pos + depth may be any number, -1 among them: the rows get what queries that come rotated get."""
    lens, theta = [50, 33], 1e4
    cache, table = tree.pool(pc, 50, 2, lens, w, 2, 16, d, fmt)
    q = _normal(51, 2, w, Hq, d)
    at = np.array([[first + i for i in range(w)], [first + 3 + i for i in range(w)]])
    border = tree.near_a_border(ref.f64(q), at, theta)                # no element that fp32 may round either way
    q[torch.from_numpy(np.concatenate([border, border], -1))] = 0
    turned = torch.from_numpy(ref.to_bf16(tree.turned(ref.f64(q), at, theta)).astype(np.float32)).to(torch.bfloat16)
    want = pc.tree_attn(turned.cuda(), cache, table, _i32(lens), want_lse=True)
    for pos, pos0 in (([first, first + 3], 0), ([0, 3], first)):
        got = pc.tree_attn(q.cuda(), cache, table, _i32(lens), pos=_i32(pos), pos0=pos0, rope_theta=theta, want_lse=True)
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


@pytest.mark.parametrize("fmt", FORMATS)
def test_one_tree_for_all_sequences(fmt):
    """page_append takes the parents that tree_attn takes: [w] for all sequences."""
    B, w, parents = 3, 6, _i32([-1, 0, 0, 1, -2, 3])
    k, v, table = _normal(70, B, w, 2, 64).cuda(), _normal(71, B, w, 2, 64).cuda(), _i32([[0, 1], [2, 3], [4, 5]])
    pools = [pc.kv_cache(6, 2, 16, 64, fmt) for _ in range(2)]
    for pool, p in zip(pools, (parents, parents.repeat(B, 1))):
        pc.page_append(pool, k, v, table, at=_i32([0, 13, 20]), parents=p, rope_theta=1e4)
    for name, x in pools[0].items():
        if torch.is_tensor(x):
            assert torch.equal(x.view(torch.uint8), pools[1][name].view(torch.uint8)) and x.view(torch.uint8).any()


WIDE = [s[:4] for s in SHAPES if s[4] == "wide"]


def _near(got, want, want_lse):
    """weights rounded to bf16 or halves: 2 * 2^-9 of sum p |v| <= 4.5, the output half a step; lse: logits in fp32"""
    there, lse = np.isfinite(want_lse), got["lse"].cpu().numpy().astype(np.float64)
    assert np.array_equal(there, np.isfinite(lse)) and (lse[~there] == -INF).all()
    assert (np.abs(ref.f64(got["out"]) - want) <= 1.8e-2 + 2.0 ** -8 * np.abs(want)).all()
    assert (np.abs(np.where(there, lse, 0) - np.where(there, want_lse, 0)) <= 1e-4 + 1e-5 * np.abs(np.where(there, want_lse, 0))).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("theta,far", [(1e4, -40), (5e5, 100000), (1e6, 2 ** 28)])
@pytest.mark.parametrize("B,w,Hq,most", WIDE)
def test_many_rows_are_rotated(fmt, theta, far, B, w, Hq, most):
    """Positions of depths in a tree, from given starts, before the first and far ones; queries out of a projection, tables and parents with a pitch."""
    d, page, lens = 128, 32, [90 + 7 * b for b in range(B)]
    cache, table = tree.pool(pc, 80, B, lens, w, 2, page, d, fmt)
    g = np.random.default_rng(81)
    parents = [[int(g.integers(max(-1, i - 4), i)) for i in range(w)] for _ in range(B)]
    pos = [far + 5 * b for b in range(B)]
    q = _normal(82, B, w, 3 * Hq, d)
    depth = np.array([[len(p) - 1 for p in tree.seen(row)] for row in parents])
    border = tree.near_a_border(ref.f64(q), np.array(pos)[:, None] + depth, theta)            # no element that fp32 may round either way
    q[torch.from_numpy(np.concatenate([border, border], -1))] = 0
    room, wide = _room(table, page, most + w), torch.full((B, w + 3), -9, dtype=torch.int32, device="cuda")
    wide[:, 2:2 + w] = _i32(parents)
    pitch = torch.full((B, room.shape[1] + 5), -3, dtype=torch.int32, device="cuda")
    pitch[:, 1:1 + room.shape[1]] = room
    got = pc.tree_attn(q.cuda()[:, :, Hq:2 * Hq], cache, pitch[:, 1:1 + room.shape[1]], _i32(lens), parents=wide[:, 2:2 + w], pos=_i32([5 * b for b in range(B)]), pos0=far,
                       rope_theta=theta, max_len=most, softmax_scale=0.11, want_lse=True)
    assert got["status"].item() == 0
    want = tree.attention(ref.f64(q[:, :, Hq:2 * Hq]), tuple(np.nan_to_num(x) for x in tree.values(cache)), table.cpu().numpy(), lens, parents, pos, theta, 0.11)
    _near(got, *want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,w,Hq,most", WIDE)
def test_many_rows_over_one_page_of_any_size(fmt, d, B, w, Hq, most):
    """A page of an odd number of entries, one for each sequence, to its last entry."""
    page = most + w + 3
    lens = [page - w, 129, 300, 0, 1, 77, 500, 128][:B]
    cache, table = tree.pool(pc, 83, B, lens, w, 2, page, d, fmt)
    q, parents = _normal(84, B, w, Hq, d), [tree.chain(w)] * B
    got = pc.tree_attn(q.cuda(), cache, table, _i32(lens), want_lse=True)
    rows = [0, w // 2, w - 1]                                          # (the longest by a few rows: the reference goes row by row)
    held = tuple(np.nan_to_num(x) for x in tree.values(cache))
    for b in range(B):
        which = rows if lens[b] > 1000 else list(range(w))
        qs = np.zeros((1, w, Hq, d))
        qs[0, which] = ref.f64(q[b])[which]
        chain = [p if any(i <= r for r in which) else -2 for i, p in enumerate(parents[b])]
        want, want_lse = tree.attention(qs, held, table[b:b + 1].cpu().numpy(), [lens[b]], [chain], [0], 0)
        part = {"out": got["out"][b:b + 1, which], "lse": got["lse"][b:b + 1][:, :, which]}
        _near(part, want[:, which], want_lse[:, :, which])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,most", WIDE)
def test_many_rows_and_what_is_no_page_or_length(fmt, B, w, Hq, most):
    """Reported, not followed, and nothing to the other sequences; zeros for a length that is none, entries of zeros for a page."""
    lens, page = [40 + 10 * b for b in range(B)], 16
    cache, table = tree.pool(pc, 85, B, lens, w, 2, page, 64, fmt)
    q, others = _normal(86, B, w, Hq, 64).cuda(), [b for b in range(B) if b != 1]
    call = lambda t, n: pc.tree_attn(q, cache, _room(t, page, most + w), _i32(n), max_len=most, want_lse=True)        # noqa: E731
    good, held = call(table, lens), tuple(np.nan_to_num(x) for x in tree.values(cache))
    for bad in (-1, -2 ** 31, cache["k"].shape[0], 2 ** 31 - 1):
        other = table.clone()
        other[1, 1] = bad
        got = call(other, lens)
        assert got["status"].item() == 421 and torch.equal(got["out"][others], good["out"][others]) and torch.equal(got["lse"][others], good["lse"][others])
    none = tuple(np.concatenate([x, np.zeros_like(x[:1])]) for x in held)
    ids = table.cpu().numpy().copy()
    ids[1, 1] = len(held[0])
    want, want_lse = tree.attention(ref.f64(q), none, ids, lens, [tree.chain(w)] * B, [0] * B, 0)
    _near(got, want, want_lse)
    for bad in (most + 1, 2 ** 31 - 1):
        got = call(table, [bad if b == 1 else n for b, n in enumerate(lens)])
        assert got["status"].item() == 422 and not got["out"][1].any() and (got["lse"][1] == -INF).all()
        assert torch.equal(got["out"][others], good["out"][others]) and torch.equal(got["lse"][others], good["lse"][others])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,most", WIDE)
def test_many_rows_again_on_any_stream_in_a_graph_with_kept_buffers(fmt, B, w, Hq, most):
    lens, page = [300 + 90 * b for b in range(B)], 16
    cache, table = tree.pool(pc, 87, B, lens, w, 2, page, 128, fmt)
    table, q, n, kept = _room(table, page, most + w), _normal(88, B, w, Hq, 128).cuda(), _i32(lens), {}
    call = lambda **kw: pc.tree_attn(q, cache, table, n, rope_theta=1e4, max_len=most, want_lse=True, **kw)            # noqa: E731
    first, side = call(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call(buffers=kept)
        pc.tree_attn(q[:1, :1], cache, table[:1], n[:1], max_len=most, buffers=kept)
        with torch.cuda.graph(graph, stream=side):
            second = call(buffers=kept)
        for _ in range(3):
            second["out"].zero_()
            graph.replay()
            third = call()                                              # (another call's memory, beside the replays)
    torch.cuda.synchronize()
    for r in (second, third):
        assert torch.equal(r["out"], first["out"]) and torch.equal(r["lse"], first["lse"]) and r["status"].item() == 0
