"""Attention of drafted tokens over paged caches against 64 bits, through the public call."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import cache_ref as ref
from tests import tree_ref as tree

pytestmark = pytest.mark.gpu
FORMATS = ["bf16", "int8", "e4m3"]
NAN, INF = float("nan"), float("inf")


def _normal(seed, *shape, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _check(got, want, what, lse, want_lse):
    """Outputs are bf16 (half a step: 2^-9 of the value) of sums whose weights, and over codes the values, were rounded to bf16 (2^-9 each of sum p |v| <= max |v|,
    some 4.5 here; many keys average it away, one key has it whole) -> |error| <= 2^-9 |ref| + 2 * 2^-9 * 4.5 = 1.8e-2 + 2^-9 |ref|, and its root mean square, where
    roundings are independent and of uniform size (0.29 of a step each), well below half of 2^-8 of the outputs'.  lse: fp32 exponentials and sums,
    and logits in fp32 (|q| |k| up to some 60 * 2^-22 after scaling): 1e-4."""
    assert np.isfinite(got).all(), what
    there = np.isfinite(want_lse)
    assert np.array_equal(there, np.isfinite(lse)) and (lse[~there] == -np.inf).all(), what
    d = np.abs(got - want)
    assert (d <= 1.8e-2 + 2.0 ** -8 * np.abs(want)).all(), (what, d.max())
    assert np.sqrt((d ** 2).mean()) <= 3.5e-3 * np.sqrt((want ** 2).mean()) + 1e-6, (what, np.sqrt((d ** 2).mean() / (want ** 2).mean()))
    assert (np.abs(lse - want_lse)[there] <= 1e-4 + 1e-5 * np.abs(want_lse[there])).all(), (what, np.abs(lse - want_lse)[there].max())


def _trees(seed, B, w, kind):
    """parents [B][w]: a chain, siblings, random trees, random trees of different sizes (-2: not there) with a token among them that is not there either"""
    g = np.random.default_rng(seed)
    if kind == "chain":
        return [tree.chain(w)] * B
    if kind == "siblings":
        return [[-1] * w] * B
    out = []
    for _ in range(B):
        p = [int(g.integers(max(-1, i - 5), i)) for i in range(w)]
        if kind == "fewer":
            there = int(g.integers(0, w + 1))
            p = [x if i < there else -2 for i, x in enumerate(p)]
            if there > 2:
                p[int(g.integers(0, there))] = -2                     # its descendants are not there either
        out.append(p)
    return out


def _run(fmt, B, w, Hq, Hkv, d, page, n, *, kind="random", ragged=False, theta=1.0e4, seed=20, scale=0.0, given_pos=False, far=0, big=1.0, max_len=None, **kwargs):
    lens = [(n * ((7 * b + 3) % 11)) // 10 for b in range(B)] if ragged else [n] * B
    if ragged and B > 4:
        lens[4] = -1                                                  # a padded batch
    cache, table = tree.pool(pc, seed, B, lens, w, Hkv, page, d, fmt, big=big)
    parents = _trees(seed + 1, B, w, kind)
    pos = [5 * b + 3 + far for b in range(B)] if given_pos else [x + far for x in lens]
    q = _normal(seed + 2, B, w, Hq, d)
    if theta:                                                         # no element that fp32 may round either way
        depth = np.array([[max(len(p) - 1, 0) for p in tree.seen(row)] for row in parents])
        border = tree.near_a_border(ref.f64(q), np.array(pos)[:, None] + depth, theta)
        q[torch.from_numpy(np.concatenate([border, border], -1))] = 0
    given = None if kind == "chain" and seed % 2 == 0 else _i32(parents)
    got = pc.tree_attn(q.cuda(), cache, table, _i32(lens), parents=given, pos=_i32([5 * b + 3 for b in range(B)]) if given_pos else None, pos0=far, rope_theta=theta,
                       softmax_scale=scale, max_len=max_len, want_lse=True, **kwargs)
    assert got["status"].item() == 0
    want, want_lse = tree.attention(ref.f64(q), tuple(np.nan_to_num(x) for x in tree.values(cache)), table.cpu().numpy(), lens, parents, pos, theta, scale)
    _check(ref.f64(got["out"]), want, "out", got["lse"].cpu().numpy().astype(np.float64), want_lse)
    return got


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,Hkv,d,page,n", [
    (1, 1, 1, 1, 64, 16, 0), (1, 1, 1, 1, 128, 16, 1), (1, 1, 8, 2, 128, 16, 15), (2, 1, 8, 2, 64, 32, 16), (2, 1, 7, 1, 128, 48, 47), (1, 1, 4, 4, 64, 64, 63),
    (3, 1, 8, 1, 128, 64, 64), (2, 1, 6, 2, 64, 128, 127), (1, 1, 10, 2, 128, 80, 129), (1, 1, 32, 8, 128, 256, 3000), (5, 1, 14, 2, 64, 112, 1001)])
def test_single_tokens(fmt, B, w, Hq, Hkv, d, page, n):
    _run(fmt, B, w, Hq, Hkv, d, page, n)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["chain", "siblings", "random", "fewer"])
@pytest.mark.parametrize("B,w,Hq,Hkv,d,page,n", [
    (1, 2, 2, 2, 64, 16, 0), (2, 3, 4, 2, 128, 16, 13), (1, 8, 2, 1, 64, 48, 100), (2, 5, 14, 2, 64, 32, 250), (3, 12, 4, 2, 128, 64, 500),
    (1, 33, 2, 2, 128, 16, 31), (2, 64, 2, 1, 64, 16, 200), (1, 64, 8, 1, 128, 128, 129), (2, 31, 8, 2, 64, 96, 300), (1, 63, 4, 4, 128, 256, 1)])
def test_trees(fmt, kind, B, w, Hq, Hkv, d, page, n):
    """New tokens across the ends of units, tiles and pages, with nothing before them too."""
    _run(fmt, B, w, Hq, Hkv, d, page, n, kind=kind, seed=30 + w)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,Hkv,d,page,n", [(11, 1, 8, 2, 128, 16, 700), (11, 4, 14, 2, 64, 48, 257), (12, 12, 8, 2, 128, 32, 1000), (7, 40, 8, 1, 64, 64, 2000),
                                                 (160, 1, 8, 2, 128, 16, 90), (160, 2, 16, 2, 64, 16, 60), (310, 1, 4, 2, 64, 32, 90)])
def test_sequences_of_different_lengths(fmt, B, w, Hq, Hkv, d, page, n):
    """Lengths from zero on, a sequence that is not there, trees of different sizes."""
    _run(fmt, B, w, Hq, Hkv, d, page, n, kind="fewer", ragged=True, given_pos=True)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("w,Hq", [(1, 8), (6, 8), (24, 8)])
def test_long_sequences_in_many_splits(fmt, w, Hq):
    _run(fmt, 1, w, Hq, 2, 128, 16, 20011, theta=5e5)
    _run(fmt, 2, w, Hq, 2, 64, 64, 9000, theta=0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("page", [1, 7, 100, 129, 1000, 3001])
@pytest.mark.parametrize("w", [1, 5, 30])
def test_sequences_of_one_page_of_any_size(fmt, page, w):
    """A cache of kv_cache(B, Hkv, capacity, ..) is a pool of one page a sequence."""
    if w <= page:
        _run(fmt, 3, w, 4, 2, 64, page, page - w, theta=0)
        _run(fmt, 3, w, 4, 2, 128, page, page - w, theta=0, ragged=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("theta,far", [(1e4, 0), (5e5, 100000), (1e6, 2 ** 30)])
def test_rotation_at_far_positions(d, theta, far):
    for w in (1, 20):
        _run("bf16", 2, w, 4, 2, d, 32, 150, theta=theta, far=far, given_pos=True)


def test_shared_pages_and_one_tree_for_all():
    """Sequences with common pages; parents [w]; a table whose rows lie apart; strided queries; a softmax scale."""
    B, w, Hq, Hkv, d, page, n = 4, 6, 8, 2, 64, 16, 64
    cache, table = tree.pool(pc, 3, 1, [n + 200], w, Hkv, page, d, "bf16", spoil=False)
    wide = torch.full((B, 9), -7, dtype=torch.int32, device="cuda")
    wide[:, 2:6] = table[0, :4]
    wide[:, 6] = table[0, 5:5 + B]
    both = _normal(4, B, w, 3 * Hq, d).cuda()
    q, parents, lens = both[:, :, Hq:2 * Hq], [-1, 0, 0, 1, 1, 2], [n, n - 3, n - 16, 10]
    got = pc.tree_attn(q, cache, wide[:, 2:7], _i32(lens), parents=_i32(parents), softmax_scale=0.3, want_lse=True)
    want, want_lse = tree.attention(ref.f64(q), tree.values(cache), wide[:, 2:7].cpu().numpy(), lens, [parents] * B, lens, 0, 0.3)
    _check(ref.f64(got["out"]), want, "out", got["lse"].cpu().numpy(), want_lse)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("w,Hq", [(5, 4), (20, 8), (60, 8)])
def test_a_token_that_is_no_number_stays_where_it_is_seen(fmt, w, Hq):
    """NaN and infinities in a drafted token's values and keys: only its descendants and itself have them, an infinity keeps its sign."""
    B, Hkv, d, page, n = 2, 2, 64, 16, 37
    lens = [n, 3]
    cache, table = tree.pool(pc, 8, B, lens, w, Hkv, page, d, fmt)
    where = lambda b, i: (int(table[b, (lens[b] + i) // page]), (lens[b] + i) % page)                    # noqa: E731
    parents = [[-1, 0, -1, 2, 3] + [3] * (w - 5), [-1, 0, 1, 0, -1] + [-1] * (w - 5)]
    q = _normal(9, B, w, Hq, d).cuda()
    clean = ref.f64(pc.tree_attn(q, cache, table, _i32(lens), parents=_i32(parents))["out"])
    p0, e0 = where(0, 2)                                                # seen by 2, 3 and all from 4 on
    p1, e1 = where(1, 1)                                                # seen by 1 and 2
    if fmt == "bf16":
        cache["v"][p0, 1, e0, 7], cache["v"][p0, 1, e0, 8], cache["k"][p1, 0, e1, 3] = INF, NAN, NAN
    else:
        cache["v_scale"][p0, 1, e0], cache["k_scale"][p1, 0, e1] = NAN, NAN
    got = ref.f64(pc.tree_attn(q, cache, table, _i32(lens), parents=_i32(parents))["out"])
    G, hit = Hq // Hkv, np.zeros(got.shape, bool)
    for i in [2] + list(range(3, w)):
        hit[0, i, G:, 8] = True
        if fmt == "bf16":
            assert np.isposinf(got[0, i, G:, 7]).all()
        else:
            hit[0, i, G:] = True
    hit[1, 1:3, :G] = True
    if fmt == "bf16":
        got[0, 2:, G:, 7] = clean[0, 2:, G:, 7]
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("w,Hq", [(5, 4), (20, 8)])
def test_codes_that_are_no_number(w, Hq):
    """NaN codes of e4m3 in a token that some do not see."""
    cache, table = tree.pool(pc, 8, 1, [20], w, 2, 32, 128, "e4m3")
    q, parents = _normal(9, 1, w, Hq, 128).cuda(), _i32([[-1, 0, -1] + [0] * (w - 3)])
    clean = ref.f64(pc.tree_attn(q, cache, table, _i32([20]), parents=parents)["out"])
    cache["v"].view(torch.uint8)[int(table[0, 0]), 1, 21, 5] = 0xFF
    got = ref.f64(pc.tree_attn(q, cache, table, _i32([20]), parents=parents)["out"])
    assert np.isnan(got[0, 1, Hq // 2:, 5]).all()
    got[0, 1, Hq // 2:, 5] = clean[0, 1, Hq // 2:, 5]
    assert np.array_equal(got, clean)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("w", [1, 20])
def test_values_that_are_no_number_before_the_tokens_reach_all(fmt, w):
    cache, table = tree.pool(pc, 10, 1, [200], w, 2, 16, 64, fmt)
    p, e = int(table[0, 5]), 9
    cache["v" if fmt == "bf16" else "v_scale"][p, 1, e] = NAN
    out = ref.f64(pc.tree_attn(_normal(11, 1, w, 4, 64).cuda(), cache, table, _i32([200]))["out"])
    assert np.isfinite(out[:, :, :2]).all() and np.isnan(out[:, :, 2:]).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_logits_that_grow_along_the_cache(fmt):
    """The reference maximum is raised again and again, and logits of hundreds."""
    for w, Hq in ((1, 8), (10, 8)):
        _run(fmt, 2, w, Hq, 2, 128, 16, 700, scale=0.2, theta=0)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq", [(2, 1, 8), (1, 6, 8), (3, 40, 8)])
def test_values_of_any_size_beside_one_another(fmt, B, w, Hq):
    """Values from 2^-20 to 2^20 and rows of zeros; keys that grow, so that the reference is raised again and again."""
    Hkv, d, page, n = 2, 128, 32, 700
    g = torch.Generator().manual_seed(40)
    pages = (n + w + page - 1) // page
    k, v = (torch.randn(pages, page, Hkv, d, generator=g) for _ in range(2))
    at = torch.arange(pages * page).view(pages, page, 1, 1)
    k, v = (k * (0.01 + 2.5 * at / n)).to(torch.bfloat16), (v * torch.exp2((at * 37 % 41 - 20).float()) * (at % 13 != 5)).to(torch.bfloat16)
    cache = {"format": "bf16", "k": k.transpose(1, 2).contiguous().cuda(), "v": v.transpose(1, 2).contiguous().cuda()}
    if fmt != "bf16":
        cache = pc.kv_cache(pages, Hkv, page, d, fmt)
        pc.kv_quantize(cache, k.cuda(), v.cuda())
    q, table = _normal(41, B, w, Hq, d), torch.arange(pages, dtype=torch.int32, device="cuda").expand(B, pages)
    got = pc.tree_attn(q.cuda(), cache, table, _i32([n] * B), want_lse=True)
    held, parents = tree.values(cache), [tree.chain(w)] * B
    want, want_lse = tree.attention(ref.f64(q), held, table.cpu().numpy(), [n] * B, parents, [0] * B, 0)
    size, _ = tree.attention(ref.f64(q), (held[0], np.abs(held[1])), table.cpu().numpy(), [n] * B, parents, [0] * B, 0)
    # weights rounded to bf16 (2^-9 each), the output once more
    assert (np.abs(ref.f64(got["out"]) - want) <= 1.01 * 2.0 ** -8 * size + 2.0 ** -8 * np.abs(want)).all()
    assert np.abs(got["lse"].cpu().numpy() - want_lse).max() <= 1e-4 + 1e-5 * np.abs(want_lse).max()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("w", [2, 30])
def test_pages_and_lengths_that_are_none(fmt, w):
    """Page ids outside the pool are not followed, lengths beyond the table or max_len are no sequences; both are reported, other sequences are right."""
    lens = [40, 40, 40]
    cache, table = tree.pool(pc, 12, 3, lens, w, 2, 16, 64, fmt)
    q = _normal(13, 3, w, 4, 64).cuda()
    want = pc.tree_attn(q, cache, table, _i32(lens))["out"]
    for bad in (-1, -2 ** 31, cache["k"].shape[0], 2 ** 31 - 1):
        other = table.clone()
        other[1, 1] = bad
        got = pc.tree_attn(q, cache, other, _i32(lens))
        assert got["status"].item() == 421
        assert torch.equal(got["out"][0], want[0]) and torch.equal(got["out"][2], want[2])
    room = table.shape[1] * 16 - w
    for bad, limit in ((room + 1, None), (2 ** 31 - 1, None), (41, 40)):
        got = pc.tree_attn(q, cache, table, _i32([40, bad, 40]), want_lse=True, max_len=limit)
        assert got["status"].item() == 422 and not got["out"][1].any() and (got["lse"][1] == -INF).all()
        assert torch.equal(got["out"][0], want[0]) and torch.equal(got["out"][2], want[2])
    got = pc.tree_attn(q, cache, table, _i32([40, -5, 40]), want_lse=True)
    assert got["status"].item() == 0 and not got["out"][1].any() and (got["lse"][1] == -INF).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_parents_that_are_none(fmt):
    """A token that follows itself, a later one or nothing that there is, is not there."""
    w = 7
    cache, table = tree.pool(pc, 14, 1, [30], w, 1, 16, 64, fmt)
    q = _normal(15, 1, w, 2, 64).cuda()
    want = pc.tree_attn(q, cache, table, _i32([30]), parents=_i32([[-1, 0, -2, 1, -2, -2, -2]]), want_lse=True)
    got = pc.tree_attn(q, cache, table, _i32([30]), parents=_i32([[-1, 0, 2, 1, 6, 2 ** 31 - 1, -2 ** 31]]), want_lse=True)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    assert (want["lse"][0, :, [2, 4, 5, 6]] == -INF).all() and torch.isfinite(want["lse"][0, :, [0, 1, 3]]).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,Hkv,n", [(3, 1, 8, 2, 900), (2, 12, 8, 2, 400), (2, 40, 8, 2, 700)])
def test_same_results_every_time_on_any_stream_in_a_graph_and_with_kept_buffers(fmt, B, w, Hq, Hkv, n):
    lens, d = [n - 17 * b for b in range(B)], 128
    cache, table = tree.pool(pc, 16, B, lens, w, Hkv, 32, d, fmt)
    q, ln, parents, kept = _normal(17, B, w, Hq, d).cuda(), _i32(lens), _i32(_trees(18, B, w, "random")), {}
    call = lambda **kw: pc.tree_attn(q, cache, table, ln, parents=parents, rope_theta=1e4, want_lse=True, **kw)          # noqa: E731
    first = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = call(buffers=kept)
        out, lse = second["out"].clone(), second["lse"].clone()
        pc.tree_attn(q[:1, :1], cache, table[:1], ln[:1], buffers=kept)                               # a smaller call has views
        third = call(buffers=kept)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fourth = call(buffers=kept)
        fourth["out"].zero_()
        graph.replay()
    torch.cuda.current_stream().wait_stream(side)
    assert kept["workspace"].data_ptr() == second["workspace"].data_ptr()
    for r in ((out, lse), (third["out"], third["lse"]), (fourth["out"], fourth["lse"])):
        assert torch.equal(r[0], first["out"]) and torch.equal(r[1], first["lse"])


def test_pages_beyond_2_31_elements():
    """The pool's last pages lie beyond 2^31 elements and bytes."""
    Hkv, d, page, w, n = 8, 128, 256, 3, 600
    small, table = tree.pool(pc, 19, 1, [n], w, Hkv, page, d, "bf16", spoil=False)
    pages = 2 ** 31 // (Hkv * page * d) + 5
    k, v = (torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    last = pages - small["k"].shape[0]
    k[last:], v[last:] = small["k"], small["v"]
    q = _normal(20, 1, w, 16, d).cuda()
    want = pc.tree_attn(q, small, table, _i32([n]))["out"]
    assert torch.equal(pc.tree_attn(q, {"format": "bf16", "k": k, "v": v}, table + last, _i32([n]))["out"], want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n,code", [(1, 1, 8, 2, 128, 1500, 411), (4, 1, 8, 2, 64, 2000, 411), (160, 1, 2, 2, 128, 70, 411),
                                                   (1, 32, 32, 8, 128, 12000, 101), (1, 32, 32, 8, 64, 12000, 101)])
def test_a_wait_that_runs_out_is_reported(fmt, B, w, Hq, Hkv, d, n, code):
    """The kernels wait for one arrival that nobody makes, with nothing in flight: 2e6 cycles, about a millisecond.  (Many rows: the message that there is no
    more work, behind the one item of each CTA.)"""
    lib = pc.load_library()
    cache, table = tree.pool(pc, 21, B, [n] * B, w, Hkv, 32, d, fmt, spoil=False)
    q, lens = _normal(22, B, w, Hq, d).cuda(), _i32([n] * B)
    clean = pc.tree_attn(q, cache, table, lens)["out"].clone()
    assert lib.pc_debug_bounded_wait_test(2_000_000, 1) == 0
    try:
        hit = pc.tree_attn(q, cache, table, lens)["status"].item()
    finally:
        assert lib.pc_debug_bounded_wait_test(0, 0) == 0
    assert hit == code
    again = pc.tree_attn(q, cache, table, lens)
    assert again["status"].item() == 0 and torch.equal(again["out"], clean)


def test_refusals():
    cache, table = pc.kv_cache(6, 2, 16, 64, "int8"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    q, lens = torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16, device="cuda"), _i32([3, 4])
    pc.tree_attn(q, cache, table, lens, max_len=44)
    for change in (dict(q=q.float()), dict(q=q[..., :32]), dict(q=q[:, :, :3]), dict(q=q[0]), dict(q=q.cpu()), dict(table=table.long()), dict(table=table[:1]),
                   dict(table=table[0]), dict(table=None), dict(table=table.t().contiguous().t()), dict(lens=None), dict(lens=_i32([1])), dict(lens=lens.float()),
                   dict(parents=_i32([[0]])), dict(parents=_i32([0] * 5)), dict(max_len=45), dict(max_len=-1), dict(rope_theta=-1.0), dict(rope_theta=INF),
                   dict(softmax_scale=-1.0), dict(softmax_scale=NAN), dict(pos=_i32([1])), dict(pos0=2 ** 31), dict(cache=dict(cache, k_scale=None)),
                   dict(cache=pc.kv_cache(6, 2, 20, 64, "int8")), dict(cache=pc.kv_cache(6, 3, 16, 64, "int8")), dict(cache=pc.kv_cache(6, 2, 16, 128, "int8")),
                   dict(q=q.repeat(1, 17, 1, 1), table=table.repeat(1, 4)), dict(out=torch.empty(2, 4, 4, 64, device="cuda")),
                   dict(table=table[:, :0]), dict(q=q.repeat(1, 13, 1, 1))):
        a = dict(dict(q=q, cache=cache, table=table, lens=lens), **change)
        with pytest.raises(pc.PcError):
            pc.tree_attn(a.pop("q"), a.pop("cache"), a.pop("table"), a.pop("lens"), **a)
