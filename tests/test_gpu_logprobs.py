"""Log probabilities, entropies and alternatives of rows of logits against 64 bits, through the public call."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import tree_ref as tree

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
INF, NAN = float("inf"), float("nan")


def _f64(t):
    return t.detach().cpu().double().numpy()


def _check(x, tokens, top, got, scale=1.0, group=0):
    """A sum of V terms in fp32: a thread adds at most V / 512 + 8 of them one by one (2^-24 each), joins 20 times, and a term is good to 2^-21: the logarithm is off by
    (V / 512 + 48) 2^-24 at most; the logit less the maximum is rounded once and scaled (2^-23 of it).  The entropy's sum has terms up to its own size."""
    want, entropy, ids, lp = tree.logprobs(_f64(x), tokens.cpu().numpy(), top, scale)
    V = x.shape[1]
    off = (V / 512 + 48) * 2.0 ** -24

    def near(a, b, tol):
        a, there = _f64(a), np.isfinite(b)
        assert np.array_equal(a[~there], b[~there], equal_nan=True)
        assert (np.abs(a - b)[there] <= tol[there]).all(), (np.abs(a - b)[there] / tol[there]).max()

    near(got["logprob"], want, off + 2.0 ** -21 * np.nan_to_num(np.abs(want), posinf=0))
    near(got["entropy"], entropy, off * (2 + 2 * np.abs(entropy)) + 2.0 ** -21 * np.abs(entropy))
    if top:
        assert np.array_equal(got["top_id"].cpu().numpy(), ids)
        near(got["top_logprob"], lp, off + 2.0 ** -21 * np.nan_to_num(np.abs(lp), posinf=0))
    if group:
        near(got["nll"], -want.reshape(-1, group).sum(-1), group * (off + 2.0 ** -21 * np.abs(want).reshape(-1, group).max(-1)) + group * 2.0 ** -24 * np.abs(want).reshape(-1, group).sum(-1))


def _rows(seed, N, V, type, pad=0, offset=0, spread=3.0):
    """rows of a larger buffer, `pad` elements between them, the first `offset` elements into it"""
    x = (torch.randn(N * (V + pad) + offset, generator=torch.Generator().manual_seed(seed)) * spread).to(TYPES[type]).cuda()
    return x[offset:].view(N, V + pad)[:, :V]


def _tokens(seed, N, V):
    return torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N,V,top,pad,offset", [
    (1, 1, 1, 0, 0), (3, 2, 2, 0, 1), (2, 7, 5, 1, 3), (5, 8, 8, 0, 0), (4, 9, 1, 0, 1), (3, 31, 20, 2, 0), (2, 32, 32, 0, 0), (7, 33, 32, 5, 1), (3, 255, 3, 0, 0),
    (2, 1000, 32, 1, 1), (1, 4096, 20, 0, 0), (1, 50001, 32, 0, 1), (9, 50001, 5, 2, 0), (700, 3000, 4, 1, 0), (1, 131072, 32, 0, 0), (40, 128256, 20, 0, 0),
    (3, 200003, 8, 0, 3)])
def test_rows_of_any_size_and_alignment(type, N, V, top, pad, offset):
    x, t = _rows(N + V, N, V, type, pad, offset), _tokens(V, N, V)
    _check(x, t, top, pc.token_logprobs(x, t, top=top, want_entropy=True))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("N", [1, 5, 2000])
def test_ties_go_to_the_lower_index(type, N):
    """Few different values, all the same value, the largest ones in one place, rising and falling rows."""
    V = 5003
    x = torch.randint(0, 4, (N, V), generator=torch.Generator().manual_seed(1)).float()
    x[0] = 2.5
    if N > 4:
        x[1] = torch.arange(V) / 64.0
        x[2] = -torch.arange(V) / 64.0
        x[3] = -4.0
        x[3, 777:777 + 40] = 5.0
        x[4] = -0.0
        x[4, 100] = 0.0
    x = x.to(TYPES[type]).cuda()
    t = _tokens(2, N, V)
    _check(x, t, 32, pc.token_logprobs(x, t, top=32, want_entropy=True))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("V", [300, 40000])
def test_the_largest_logits_in_few_places(type, V):
    """All of the largest ones where one thread reads them: every 256th piece of 16 bytes, and pieces side by side."""
    x = torch.randn(3, V, generator=torch.Generator().manual_seed(3)).to(TYPES[type])
    per = 16 // x.element_size()
    for j in range(0, V, 256 * per):
        x[0, j:j + per] = 30.0 + torch.arange(len(x[0, j:j + per])).to(x.dtype) / 8
    x[1, V // 2:V // 2 + 100] = 20.0 + torch.arange(100) % 7
    x = x.cuda()
    t = _tokens(4, 3, V)
    _check(x, t, 32, pc.token_logprobs(x, t, top=32, want_entropy=True))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("V", [10, 9000])
def test_masked_logits(type, V):
    """-inf and the type's lowest value in most places, in all but one, in all; one large logit; tokens that are masked."""
    low = torch.finfo(TYPES[type]).min
    x = torch.randn(8, V, generator=torch.Generator().manual_seed(5))
    x[0, 3:] = -INF
    x[1, 3:] = low
    x[2] = -INF
    x[3] = low
    x[4] = -INF
    x[4, V - 1] = 1.5
    x[5] = low
    x[5, V // 2] = 2.0
    x[6, 1] = 300.0
    x[7] = -INF
    x[7, 4] = low
    x = x.to(TYPES[type]).cuda()
    for t in (_tokens(6, 8, V), torch.full((8,), V - 1, dtype=torch.int32, device="cuda"), torch.full((8,), 1, dtype=torch.int32, device="cuda")):
        _check(x, t, min(V, 12), pc.token_logprobs(x, t, top=min(V, 12), want_entropy=True))


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("at", [0, 5, 8999])
def test_rows_that_have_no_probabilities(type, bad, at):
    x = _rows(7, 3, 9000, type)
    want = pc.token_logprobs(x, _tokens(8, 3, 9000), top=4, want_entropy=True)
    x[1, at] = bad
    got = pc.token_logprobs(x, _tokens(8, 3, 9000), top=4, want_entropy=True)
    for n in want:
        if want[n] is not None:
            assert torch.equal(got[n][0], want[n][0]) and torch.equal(got[n][2], want[n][2])
    assert torch.isnan(got["logprob"][1]) and torch.isnan(got["entropy"][1]) and torch.isnan(got["top_logprob"][1]).all() and (got["top_id"][1] == -1).all()


@pytest.mark.parametrize("scale", [0.01, 1.0 / 0.7, 40.0])
def test_a_temperature(scale):
    x, t = _rows(9, 6, 20011, "bf16"), _tokens(10, 6, 20011)
    _check(x, t, 10, pc.token_logprobs(x, t, top=10, want_entropy=True, scale=scale), scale)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-20, 1e6, 1e30, 2.0 ** 100])
def test_temperatures_far_from_one(type, scale):
    """Scaled logits that are all the same to fp32, and ones whose products with scale * log2 e pass the largest number (a greedy choice by temperature)."""
    x, t = _rows(24, 5, 9001, type), _tokens(25, 5, 9001)
    x[1] *= 50.0
    x[2, 4000] = 6e4
    if type != "fp16":
        x[3] = (x[3].float() * 1e9).to(x.dtype)
        x[4] = (x[4].float() * 1e37).to(x.dtype)
    x, (want, entropy, ids, lp) = x.contiguous(), tree.logprobs(_f64(x), t.cpu().numpy(), 6, float(np.float32(scale)))
    got = pc.token_logprobs(x, t, top=6, want_entropy=True, scale=scale)
    assert np.array_equal(got["top_id"].cpu().numpy(), ids)
    # as in _check; what is below the lowest number is -inf, and where the largest logit is alone the entropy's sum is less than the least number
    for a, b in ((got["logprob"], want), (got["top_logprob"], lp), (got["entropy"], entropy)):
        a, far = _f64(a), np.abs(b) > 3.4e38
        assert np.isneginf(a[far]).all() and not np.isnan(a).any()
        assert (np.abs(a - b)[~far] <= ((9001 / 512 + 48) * 2.0 ** -24 * (2 + 2 * np.minimum(np.abs(b), 20)) + 2.0 ** -21 * np.abs(b))[~far]).all()


def test_logits_that_lie_further_apart_than_the_largest_number():
    x = torch.full((2, 5000), -3e38, device="cuda")
    x[:, 17], x[1, 4999] = 3e38, 2.9e38
    got = pc.token_logprobs(x, torch.tensor([3, 4999], dtype=torch.int32, device="cuda"), top=2, scale=0.125, want_entropy=True)
    assert got["top_id"].tolist() == [[17, 0], [17, 4999]] and got["top_logprob"][:, 0].tolist() == [0.0, 0.0] and got["entropy"].tolist() == [0.0, 0.0]
    want = -(torch.tensor([6e38, 0.1e38], dtype=torch.float64) * 0.125)
    assert ((got["logprob"].cpu().double() - want).abs() <= 2.0 ** -18 * want.abs()).all()          # (the second: a difference of two that are rounded, 2^-24 of 3e38)


def test_groups_and_tokens_that_are_none():
    """Sums over groups, a row that adds nothing, a token behind the last; what is not asked for is not there."""
    C, w, V = 5, 37, 3001
    x, t = _rows(11, C * w, V, "bf16"), _tokens(12, C * w, V)
    t[3], t[40] = -1, -2 ** 31
    got = pc.token_logprobs(x, t, group=w, want_entropy=True)
    _check(x, t, 0, got, group=w)
    assert got["top_id"] is None and got["logprob"][3] == 0
    again = pc.token_logprobs(x, t, group=w)
    assert again["entropy"] is None and torch.equal(again["nll"], got["nll"])
    t[5] = V
    assert torch.isnan(pc.token_logprobs(x, t)["logprob"][5])
    only = pc.token_logprobs(x, top=3)
    assert only["logprob"] is None and torch.equal(only["top_id"], pc.token_logprobs(x, t, top=3)["top_id"])


def test_one_row_for_all():
    x, t = _rows(13, 1, 700, "fp32").expand(6, 700), _tokens(14, 6, 700)
    _check(x, t, 7, pc.token_logprobs(x, t, top=7, want_entropy=True))


def test_chunk_scores_of_the_path():
    """Eq. 3: the self-information of the query window behind every chunk ranks the chunks of hot_path."""
    C, L, w, Hq, Hkv, d, V, m = 5, 96, 16, 4, 2, 64, 2000, 2
    g = torch.Generator().manual_seed(15)
    q, k, v = ((torch.randn(C, L, h, d, generator=g)).to(torch.bfloat16).cuda() for h in (Hq, Hkv, Hkv))
    logits, window = _rows(16, C * w, V, "bf16"), _tokens(17, w, V)
    score = pc.token_logprobs(logits, window.repeat(C), group=w)["nll"]
    kept = pc.hot_path(q, k, v, w=w, rope_theta=1e4, m=m, k_keep=20, chunk_score=score)["kept"]
    lp = torch.log_softmax(logits.double().cpu().view(C, w, V), -1)
    info = -lp.gather(2, window.cpu().long().view(1, w, 1).expand(C, w, 1)).sum((1, 2))
    assert kept.tolist() == sorted(info.argsort()[:m].tolist())


def test_on_another_stream_and_in_a_graph():
    x, t = _rows(18, 30, 30011, "fp16", 1), _tokens(19, 30, 30011)
    want = pc.token_logprobs(x, t, top=8, group=10, want_entropy=True)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = pc.token_logprobs(x, t, top=8, group=10, want_entropy=True)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)


def test_rows_beyond_2_31_elements():
    V, N = 200_000, 11_000
    x = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    x[-1] = _rows(20, 1, V, "bf16")
    t = _tokens(21, N, V)
    got = pc.token_logprobs(x, t, top=5, want_entropy=True)
    _check(x[-1:], t[-1:], 5, {n: y if y is None else y[-1:] for n, y in got.items()})
    assert (got["top_id"][:-1] == torch.arange(5, device="cuda")).all() and (got["logprob"][:-1] + np.log(V)).abs().max() < 1e-4


def test_refusals():
    x, t = _rows(22, 4, 100, "fp32"), _tokens(23, 4, 100)
    for args, kwargs in [((x,), {}), ((x[0],), dict(top=1)), ((x.double(), t), {}), ((x.t(), _tokens(1, 100, 4)), {}), ((x, t.long()), {}), ((x, t[:3]), {}), ((x, t), dict(top=33)),
                         ((x[:, :5], t), dict(top=6)), ((x, t), dict(top=-1)), ((x, t), dict(group=3)), ((x,), dict(group=2, top=1)), ((x, t), dict(scale=0.0)),
                         ((x, t), dict(scale=-1.0)), ((x, t), dict(scale=INF)), ((x, t), dict(scale=NAN)), ((x.cpu(), t.cpu()), {}), ((x, t.cpu()), {}), ((x[:0], t[:0]), {})]:
        with pytest.raises(pc.PcError):
            pc.token_logprobs(*args, **kwargs)
