"""hivis_logprobs against its definition in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _to(x, dtype):
    t = _torch()
    return t.from_numpy(np.ascontiguousarray(x, np.float32)).to(t.bfloat16 if dtype == "bf16" else t.float32).cuda()


def _want(x, ids, temperature, top_n):
    """x [n, V] float64 -> (log p of ids, entropy, top ids, their log p)."""
    n, V = x.shape
    lp = np.full((n, ids.shape[1]), -np.inf)
    h, tid, tlp = np.zeros(n), np.full((n, top_n), -1), np.full((n, top_n), -np.inf)
    for r in range(n):
        ok = np.flatnonzero(x[r] > -np.inf)
        if not ok.size:
            continue
        y = x[r, ok] / temperature
        m = y.max()
        e = np.exp(y - m)
        log_z = m + math.log(e.sum())
        full = np.full(V, -np.inf)
        full[ok] = y - log_z
        p = np.exp(full[ok])
        h[r] = -(p[p > 0] * full[ok][p > 0]).sum()
        for i, t in enumerate(ids[r]):
            if 0 <= t < V:
                lp[r, i] = full[t]
        order = ok[np.lexsort((ok, -x[r, ok]))][:top_n]
        tid[r, :order.size], tlp[r, :order.size] = order, full[order]
    return lp, h, tid, tlp


def _check(x, ids, temperature, top_n, out):
    got = [None if g is None else g.double().cpu().numpy() if g.is_floating_point() else g.cpu().numpy() for g in out]
    x = x.double().cpu().numpy()
    lp, h, tid, tlp = _want(x, ids.cpu().numpy(), float(np.float32(temperature)), top_n)
    # y is one fp32 operation from exact numbers (2^-24 of itself) with a factor rounded to 2^-24, 2^y good to 2^-22, its sums
    # added up in fp32 in threads' and trees' parts (of a positive sum: 2^-19 at these lengths); the result rounded to 2^-24
    worst = np.abs(np.where(np.isfinite(x), x, 0)).max(-1, keepdims=True) / temperature
    tol = 2.0 ** -19 + 2.0 ** -22 * worst
    for g, w, t in ((got[0], lp, tol), (got[3], tlp, tol)):
        if g is None:
            continue
        assert np.array_equal(np.isneginf(g), np.isneginf(w))
        f = np.isfinite(w)
        assert np.all((np.abs(np.where(f, g - np.where(f, w, 0), 0)) <= t + 2.0 ** -23 * np.abs(np.where(f, w, 0))))
    if got[1] is not None:
        # the entropy's second sum has terms up to 1/e log2 of the vocabulary
        assert np.all(np.abs(got[1] - h) <= 2.0 ** -18 * (1 + h) + 2.0 ** -21 * worst[:, 0])
    if got[2] is not None:
        assert np.array_equal(got[2], tid)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 31, 257, 1024, 3001, 5031, 32000, 50257, 152064])
@pytest.mark.parametrize("top_n", [0, 1, 5, 32])
def test_rows_of_any_length(dtype, V, top_n):
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(V + top_n)
    n = 3 if V > 20000 else 9
    x = _to(rng.standard_normal((n, V)) * rng.uniform(0.3, 6, (n, 1)), dtype)
    ids = t.from_numpy(rng.integers(0, V, (n, 3)).astype(np.int32)).cuda()
    for temperature in (1.0, 0.6):
        _check(x, ids, temperature, top_n, logprobs(x, ids, temperature=temperature, top_n=top_n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,ld", [(1000, 1001), (1000, 1003), (5031, 5040), (5031, 6001), (33, 100)])
def test_rows_that_are_not_aligned(dtype, V, ld):
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(V)
    wide = _to(rng.standard_normal((17, ld)) * 3, dtype)
    wide[:, V:] = 1e4 if V < ld else 0                               # what lies between the rows is not theirs
    x = wide[:, :V]
    ids = t.from_numpy(rng.integers(0, V, (17, 2)).astype(np.int32)).cuda()
    _check(x, ids, 1.0, 7, logprobs(x, ids, top_n=7))


@pytest.mark.parametrize("rows", [1, 2, 147, 149, 1000, 33000])
def test_any_number_of_rows(rows):
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(rows)
    x = _to(rng.standard_normal((rows, 130)) * 2, "bf16")
    ids = t.from_numpy(rng.integers(0, 130, (rows, 1)).astype(np.int32)).cuda()
    out = logprobs(x, ids, top_n=3)
    keep = np.linspace(0, rows - 1, min(rows, 300)).astype(np.int64)
    sub = t.from_numpy(keep).cuda()
    _check(x[sub], ids[sub], 1.0, 3, [o[sub] for o in out])


def test_equal_logits_go_by_the_lowest_token():
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(1)
    V = 40000
    x = np.zeros((8, V))
    x[1] = rng.integers(0, 3, V)                                     # a third of all tokens share the largest value
    x[2, V - 1] = 1.0
    x[3] = np.where(np.arange(V) % 2, 0.0, -0.0)                     # zeros of both signs are equal
    x[4] = np.minimum(np.arange(V), 100)                             # nearly all are equal and largest
    x[5] = -np.minimum(np.arange(V), 100)
    x[6] = np.arange(V) % 200
    x[7] = rng.permutation(V) * 1e-3
    for dtype in ("bf16", "f32"):
        d = _to(x, dtype)
        ids = t.zeros((8, 1), dtype=t.int32, device="cuda")
        for top_n in (1, 20, 32):
            _check(d, ids, 1.0, top_n, logprobs(d, ids, top_n=top_n))


@pytest.mark.parametrize("V", [100, 9001, 152064])
def test_banned_tokens(V):
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(2)
    x = rng.standard_normal((7, V)) * 4
    x[0, rng.random(V) < 0.5] = -np.inf
    x[1, 3:] = -np.inf                                               # three tokens are left
    x[2, :V - 1] = -np.inf                                           # the last one alone
    x[3] = -np.inf                                                   # none
    x[4, 1::2] = -np.inf
    x[5] = -3e4                                                      # a row of the lowest useful values is no masked row
    x[6, : V // 2] = -1e30
    ids = np.stack([rng.integers(0, V, 7), np.full(7, V - 1), np.full(7, -1), np.full(7, V), np.zeros(7)], 1).astype(np.int32)
    for dtype in ("bf16", "f32"):
        d = _to(x, dtype)
        i = t.from_numpy(ids).cuda()
        out = logprobs(d, i, top_n=20)
        keep = t.tensor([0, 1, 2, 3, 4, 5], device="cuda")
        _check(d[keep], i[keep], 1.0, 20, [o[keep] for o in out])
        # -1e30 is far below everything: like a banned token for sums, an alternative all the same
        assert bool(t.isfinite(out.entropy).all()) and bool(t.isfinite(out.top_logprobs[6]).all())


def test_the_lowest_value_of_the_type_as_a_mask():
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    for dtype in (t.bfloat16, t.float32):
        x = t.full((2, 5000), t.finfo(dtype).min, dtype=dtype, device="cuda")
        x[0, 17] = 1.0
        x[0, 4000] = 0.0
        out = logprobs(x, t.tensor([[17], [3]], dtype=t.int32, device="cuda"), top_n=2)
        want = -math.log(1 + math.exp(-1))
        assert abs(float(out.logprobs[0, 0]) - want) < 1e-6 and out.top_ids[0].tolist() == [17, 4000]
        # a row of that value alone is flat
        assert abs(float(out.logprobs[1, 0]) + math.log(5000)) < 1e-5 and abs(float(out.entropy[1]) - math.log(5000)) < 1e-5
        assert out.top_ids[1].tolist() == [0, 1]


def test_rows_that_are_not_finite():
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    for dtype in (t.bfloat16, t.float32):
        x = t.randn((4, 20000), device="cuda").to(dtype)
        clean = logprobs(x, t.zeros((4, 1), dtype=t.int32, device="cuda"), top_n=3)
        x[1, 777] = math.nan
        x[2, 5] = math.inf
        out = logprobs(x, t.zeros((4, 1), dtype=t.int32, device="cuda"), top_n=3)
        for r in (1, 2):
            assert math.isnan(float(out.logprobs[r, 0])) and math.isnan(float(out.entropy[r]))
        assert out.top_ids[1].tolist() == clean.top_ids[1].tolist() or 777 in clean.top_ids[1].tolist()
        assert int(out.top_ids[2, 0]) == 5
        for r in (0, 3):
            assert all(t.equal(a[r], b[r]) for a, b in zip(out, clean))


def test_what_is_not_asked_for():
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    x = t.randn((5, 999), device="cuda")
    ids = t.randint(0, 999, (5, 2), dtype=t.int32, device="cuda")
    whole = logprobs(x, ids, top_n=4)
    assert logprobs(x).logprobs is None and t.equal(logprobs(x).entropy, whole.entropy)
    part = logprobs(x, ids, entropy=False)
    assert part.entropy is None and part.top_ids is None and t.equal(part.logprobs, whole.logprobs)
    assert t.equal(logprobs(x, top_n=4, entropy=False).top_ids, whole.top_ids)
    many = t.randint(0, 999, (5, 32), dtype=t.int32, device="cuda")
    _check(x, many, 1.0, 0, logprobs(x, many))
    assert logprobs(x[:0], ids[:0]).logprobs.shape == (0, 2)


def test_the_same_call_gives_the_same_bits_and_replays():
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    x = (t.randn((40, 32000), device="cuda") * 3).bfloat16()
    ids = t.randint(0, 32000, (40, 1), dtype=t.int32, device="cuda")
    first = logprobs(x, ids, top_n=20)
    for _ in range(3):
        assert all(t.equal(a, b) for a, b in zip(logprobs(x, ids, top_n=20), first))
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        out = logprobs(x, ids, top_n=20)
    for seed in range(3):
        x.copy_((t.randn((40, 32000), device="cuda") * (seed + 1)).bfloat16())
        graph.replay()
        got = [o.clone() for o in out]
        assert all(t.equal(a, b) for a, b in zip(got, logprobs(x, ids, top_n=20)))


def test_rows_beyond_four_gigabytes():
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    x = t.zeros((2, 3_000_000_000), dtype=t.bfloat16, device="cuda")[:, :4096]      # the second row starts 6 GB on
    x[1] = t.randn(4096, device="cuda").bfloat16()
    ids = t.tensor([[1], [2]], dtype=t.int32, device="cuda")
    _check(x, ids, 1.0, 3, logprobs(x, ids, top_n=3))


def test_tensors_that_do_not_fit_are_refused():
    from paper_2509_23928_b200 import HivisError, logprobs
    t = _torch()
    x = t.randn((3, 50), device="cuda")
    for call in (lambda: logprobs(x[0]), lambda: logprobs(x.t()), lambda: logprobs(x, t.zeros((3, 1), device="cuda")),
                 lambda: logprobs(x, t.zeros((2, 1), dtype=t.int32, device="cuda")), lambda: logprobs(x.cpu())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        logprobs(x.half())
    for kw in (dict(top_n=33), dict(temperature=0.0), dict(entropy=False)):
        with pytest.raises(HivisError):
            logprobs(x, **kw)


# ------------------------------------------------------------------------------------------- every temperature that is taken
def _check_far(x, ids, temperature, top_n, out):
    """As _check, with bounds that go by a token's own distance from the row's largest logit: log2(e) / T is rounded to 2^-24 of itself, and
    so is y, its distance in powers of two; the sums, of terms good to 2^-22, to 2^-19.  The entropy moves by that factor's error times
    the variance of log p, which the mean of its square bounds."""
    x = x.double().cpu().numpy()
    # (distances from the largest logit first: beside x / T of 1e60 a logarithm is lost even in 64 bits)
    top = np.where(np.isneginf(x).all(-1, keepdims=True), 0.0, x.max(-1, keepdims=True))
    T = float(np.float32(temperature))
    lp, h, tid, tlp = _want(x - top, ids.cpu().numpy(), T, top_n)
    with np.errstate(all="ignore"):
        for got, want in ((out.logprobs, lp), (out.top_logprobs, tlp)):
            g = got.double().cpu().numpy()
            below = want < -3.5e38                                   # beyond fp32's range, or without mass
            assert np.all(np.isneginf(g[below])) and not np.isnan(g).any()
            d = np.abs(g - want)[~below]
            assert np.all(d <= 2.0 ** -19 + 2.0 ** -21 * np.abs(want[~below])), float(d.max())
        got = out.entropy.double().cpu().numpy()
        for r in range(x.shape[0]):
            ok = x[r] > -np.inf
            y = x[r, ok] / T
            y = y - y.max() if ok.any() else y
            p = np.exp(y) / np.exp(y).sum() if ok.any() else y
            square = (p[p > 0] * np.log(p[p > 0]) ** 2).sum()
            assert abs(got[r] - h[r]) <= 2.0 ** -18 * (1 + h[r]) + 2.0 ** -22 * square, (r, got[r], h[r])
    assert np.array_equal(out.top_ids.cpu().numpy(), tid)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [1.1e-30, 1e-29, 1e-20, 1e-12, 1e-9, 3e-9, 1e-3, 1e3, 1e8, 1e20, 1e22, 1e25, 1e28, 1e29, 9e29])
@pytest.mark.parametrize("V,ld", [(200, 200), (5031, 6001), (50257, 50257)])
def test_banned_tokens_at_any_temperature(dtype, temperature, V, ld):
    """Rows whose largest logit is 0, next to 0 or far from it, with tokens at -infinity or at finite values as low."""
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(V)
    lowest = float(t.finfo(t.bfloat16 if dtype == "bf16" else t.float32).min)
    x = rng.standard_normal((12, ld)) * 4
    x[:8] -= x[:8, :V].max(-1, keepdims=True)                        # rows of log-probabilities, nearly
    some = rng.random(ld) < 0.4
    x[0, some] = -np.inf
    x[1, :V // 2] = -np.inf                                          # whole threads and whole CTAs without a token
    x[2, V // 2:] = -np.inf
    x[3, some] = lowest
    x[4, some] = -1e30
    x[5, 1::2] = -np.inf
    x[6, 3:] = -np.inf                                               # three tokens are left
    x[7, :V - 1] = -np.inf                                           # the last one alone
    x[7, V - 1] = 0.05
    x[8, some] = -np.inf
    x[9] = -np.inf
    x[10] = lowest                                                   # a row of the lowest value alone is flat
    d = _to(x, dtype)
    d[11, V // 2:] = lowest
    d = d[:, :V]
    ids = t.from_numpy(np.concatenate([rng.integers(0, V, (12, 3)), np.full((12, 1), V - 1), np.zeros((12, 1))], 1).astype(np.int32)).cuda()
    _check_far(d, ids, temperature, 7, logprobs(d, ids, temperature=temperature, top_n=7))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_views_that_start_anywhere(dtype):
    """A prompt is scored: the rows of one position, the tokens of the next; rows and tokens from the second one on."""
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    rng = np.random.default_rng(4)
    V = 50257
    x = _to(rng.standard_normal((6, V)) * 3, dtype)
    tokens = t.from_numpy(rng.integers(0, V, 6).astype(np.int32)).cuda()
    for logits, ids in ((x[:-1], tokens[1:].view(-1, 1)), (x[1:], tokens[1:].view(-1, 1)), (x[3:], tokens[3:].view(-1, 1)),
                        (x.view(2, 3, V)[:, -1], tokens[2:4].view(-1, 1)), (x[:, 5:1000], tokens[:6].view(-1, 1) % 995)):
        _check(logits, ids, 1.0, 4, logprobs(logits, ids, top_n=4))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 20000, 152064])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_every_answer_of_a_row_that_is_not_finite_is_nan(dtype, V, bad):
    """Tokens without mass too, and ids outside the vocabulary; in the rows beside it those are -infinity."""
    from paper_2509_23928_b200 import logprobs
    t = _torch()
    x = _to(np.random.default_rng(6).standard_normal((3, V)), dtype)
    x[:, 7] = -math.inf
    x[1, V - 3] = bad
    ids = t.tensor([[7, -1, V, 5]] * 3, dtype=t.int32, device="cuda")
    out = logprobs(x, ids, top_n=2)
    assert bool(out.logprobs[1].isnan().all()) and bool(out.entropy[1].isnan()) and bool(out.top_logprobs[1].isnan().all())
    for r in (0, 2):
        assert bool(out.logprobs[r, :3].isneginf().all()) and bool(t.isfinite(out.logprobs[r, 3])) and bool(t.isfinite(out.top_logprobs[r]).all())
