"""The 4-bit cache against its definition in 64 bits: rows in, rows out, and the attention over them."""
import math

import numpy as np
import pytest

from tests import kv4_reference as ref

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def _to(x, dtype):
    t = _torch()
    return t.from_numpy(np.ascontiguousarray(x, np.float32)).to(t.bfloat16 if dtype == "bf16" else t.float32).cuda()


def _np(x):
    return x.float().cpu().numpy().astype(np.float64)


def _ints(x):
    return _torch().tensor([int(i) for i in x], dtype=_torch().int32, device="cuda")


def _all_rows(cache):
    """[K, V], each [slots, max_len, heads, dh]: what every row of the cache stands for, written or not."""
    n, L = cache.n_slots, cache.max_len
    k, v = cache.read([L * i for i in range(n + 1)], _ints([0] * n))
    return [x.cpu().numpy().reshape(n, L, cache.n_kv_heads, cache.head_dim) for x in (k, v)]


def _bytes(cache):
    return [cache.data.cpu().numpy().copy()]


def _cache(*a):
    from paper_2509_23928_b200 import Kv4Cache
    return Kv4Cache(*a)


def _starts(n):
    return [0] + [int(x) for x in np.cumsum(n)]


# ---------------------------------------------------------------------------------------------- rows in, rows out
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,heads,counts,start", [
    (128, 3, [1], [0]), (128, 3, [1], [7]), (64, 5, [1, 1, 1], [0, 1, 30]), (128, 2, [2, 3, 16, 33, 0, 5], [1, 0, 15, 31, 4, 59]),
    (64, 1, [64, 17, 1, 40], [0, 47, 63, 1]), (128, 32, [3, 2], [0, 61]),
])
def test_rows_are_held_as_the_format_says(dtype, dh, heads, counts, start):
    t = _torch()
    rng = np.random.default_rng(5)
    cu = _starts(counts)
    B, total = len(counts), cu[-1]
    cache = _cache(B + 1, heads, dh, 64)
    slots = list(range(B, 0, -1))                                    # any order; slot 0 is not listed
    k, v = (_to(rng.standard_normal((total, heads, dh)) * 3 + rng.standard_normal((1, heads, dh)), dtype) for _ in range(2))
    old = _to(rng.standard_normal((64 * (B + 1), heads, dh)), "bf16")
    cache.append(old, old, [64 * i for i in range(B + 2)], _ints([0] * (B + 1)))
    before = _all_rows(cache)
    cache.append(k, v, cu, _ints(start), slots)
    k2, v2 = cache.read(cu, _ints(start), slots)
    t.cuda.synchronize()
    for got, x in ((k2, k), (v2, v)):
        want = ref.values(*ref.quantise(_np(x)))
        # m + s n is one fp32 operation on exact numbers: half a step of fp32
        assert np.all(np.abs(_np(got) - want) <= 2.0 ** -24 * np.abs(want))
    # nothing else has moved
    touched = np.zeros((B + 1, 64), bool)
    for b in range(B):
        touched[slots[b], start[b]:start[b] + counts[b]] = True
    for a, z in zip(before, _all_rows(cache)):
        assert np.array_equal(a[~touched], z[~touched])


def test_a_row_at_a_time_is_the_same_as_all_at_once():
    t = _torch()
    rng = np.random.default_rng(6)
    k, v = (_to(rng.standard_normal((45, 2, 128)), "bf16") for _ in range(2))
    whole, single = _cache(1, 2, 128, 64), _cache(1, 2, 128, 64)
    whole.append(k, v, [0, 45], _ints([3]))
    for i in rng.permutation(45):
        single.append(k[i:i + 1], v[i:i + 1], [0, 1], _ints([3 + i]))
    t.cuda.synchronize()
    for a, b in zip(_bytes(whole), _bytes(single)):
        assert np.array_equal(a, b)


def test_rows_behind_the_cache_are_dropped():
    t = _torch()
    rng = np.random.default_rng(7)
    k, v = (_to(rng.standard_normal((40, 2, 64)), "bf16") for _ in range(2))
    cache = _cache(4, 2, 64, 32)
    before = _all_rows(cache)
    cache.append(k, v, [0, 10, 20, 30, 40], _ints([27, -1, 32, 2 ** 31 - 1]))
    t.cuda.synchronize()
    for a, z in zip(before, _all_rows(cache)):
        assert np.array_equal(a[1:], z[1:]) and np.array_equal(a[0, :27], z[0, :27])
    got, _ = cache.read([0, 5], _ints([27]))
    want = ref.values(*ref.quantise(_np(k[:5])))
    assert np.all(np.abs(_np(got) - want) <= 2.0 ** -24 * np.abs(want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_that_are_hard_to_hold(dtype):
    """Ties, equal values, zeros of both signs, one far value, denormals, the ends of the range, and what is not finite."""
    rng = np.random.default_rng(8)
    rows = []
    for step in (1.0, 0.5, 3.0, 2.0 ** -100, 2.0 ** 90):
        # whole and half steps above the smallest value, both ends among them: every half is a tie
        g = rng.integers(0, 31, 32) * 0.5
        g[0], g[1] = 0.0, 15.0
        rows.append((g + 1.0) * step)
    rows.append(np.full(32, 0.3))
    rows.append(np.zeros(32))
    rows.append(np.where(np.arange(32) % 2, 0.0, -0.0))
    rows.append(np.where(np.arange(32) == 5, 1e4, rng.standard_normal(32)))
    rows.append(np.where(np.arange(32) == 5, 1.0, -1e-20 * np.arange(32)))
    rows.append(rng.standard_normal(32) * 1e-39)
    rows.append(rng.standard_normal(32) * 2.0 ** -133)
    rows.append(np.linspace(-1.5e38, 1.6e38, 32))
    rows.append(np.where(np.arange(32) == 9, np.nan, 1.0))
    rows.append(np.where(np.arange(32) == 9, np.inf, 1.0))
    rows.append(np.where(np.arange(32) == 9, -np.inf, 1.0))
    rows.append(np.where(np.arange(32) % 2, -3e38, 3e38))           # the range overflows
    x = np.stack(rows).astype(np.float32)
    k = _to(x[:, None].repeat(2, 1).reshape(len(rows), 1, 64), dtype)
    cache = _cache(1, 1, 64, 32)
    cache.append(k, k.flip(0).contiguous(), [0, len(rows)], _ints([1]))
    got_k, got_v = cache.read([0, len(rows)], _ints([1]))
    want = ref.values(*ref.quantise(_np(k)))
    for got, w in ((got_k, want), (got_v, want[::-1])):
        g = got.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(g), np.isnan(w))
        d = np.abs(g - w)
        # (half a step of fp32, which below its normal numbers is 2^-150)
        assert np.all(d[~np.isnan(d)] <= np.maximum(2.0 ** -24 * np.abs(w), 2.0 ** -150)[~np.isnan(d)])


def test_many_values_take_the_nearest_code():
    """A million fp32 values: the short form of the division must never decide what it cannot see."""
    rng = np.random.default_rng(9)
    x = rng.standard_normal((2048, 4, 128)) * np.exp(rng.uniform(-5, 5, (2048, 4, 1)))
    k, v = _to(x, "f32"), _to(np.round(x, 2), "bf16").float()
    cache = _cache(1, 4, 128, 2048)
    cache.append(k, v, [0, 2048], _ints([0]))
    got_k, got_v = cache.read([0, 2048], _ints([0]))
    for got, src in ((got_k, k), (got_v, v)):
        want = ref.values(*ref.quantise(src.cpu().numpy().astype(np.float64)))
        assert np.all(np.abs(_np(got) - want) <= 2.0 ** -24 * np.abs(want))


def test_rows_with_a_stride():
    t = _torch()
    rng = np.random.default_rng(10)
    both = _to(rng.standard_normal((21, 5 * 64)), "bf16")           # q | k | v of one projection, say
    k, v = both[:, 64:192].view(21, 2, 64), both[:, 192:].view(21, 2, 64)
    cache = _cache(1, 2, 64, 32)
    cache.append(k, v, [0, 21], _ints([4]))
    got_k, got_v = cache.read([0, 21], _ints([4]))
    t.cuda.synchronize()
    for got, x in ((got_k, k), (got_v, v)):
        want = ref.values(*ref.quantise(_np(x)))
        assert np.all(np.abs(_np(got) - want) <= 2.0 ** -24 * np.abs(want))


# ---------------------------------------------------------------------------------------------- attention
class Filled:
    """A cache with rows in it, what they stand for, and queries."""

    def __init__(self, dtype, dh, Hkv, G, lens, n_q, seed=0, max_len=None, slots=None, q_std=1.5, fill=None, spread=0.0):
        rng = np.random.default_rng(seed)
        self.rng, self.dtype, self.lens, self.n_q, self.dh, self.Hkv, self.G = rng, dtype, list(lens), n_q, dh, Hkv, G
        B = len(lens)
        self.slots = slots
        self.cache = _cache(B if slots is None else max(slots) + 1, Hkv, dh, max_len or max(max(lens), 1))
        if fill is not None:                                          # what lies in the cache where no row was put
            self.cache.data.fill_(fill)
        total = sum(lens)
        k = rng.standard_normal((total, Hkv, dh)) + 2.0 * rng.standard_normal((1, Hkv, dh))
        v = rng.standard_normal((total, Hkv, dh)) * np.exp(spread * rng.uniform(-1, 1, (total, Hkv, 1)))
        self.k, self.v = _to(k, dtype), _to(v, dtype)
        self.q = _to(rng.standard_normal((B * n_q, Hkv * G, dh)) * q_std, dtype)
        self.rows = _ints(lens)

    def put(self):
        self.cache.append(self.k, self.v, _starts(self.lens), _ints([0] * len(self.lens)), self.slots)

    def check(self, out, mask=None, mask_rows=0):
        cu = _starts(self.lens)
        got, q = _np(out).reshape(len(self.lens), self.n_q, self.Hkv * self.G, self.dh), _np(self.q).reshape(len(self.lens), self.n_q, -1, self.dh)
        scale = self.dh ** -0.5
        for b, L in enumerate(self.lens):
            kq, vq = ref.quantise(_np(self.k[cu[b]:cu[b + 1]])), ref.quantise(_np(self.v[cu[b]:cu[b + 1]]))
            see = ref.visible(L, self.n_q, None if mask is None else mask[b], mask_rows)
            want, reach, big = ref.attention(q[b], kq, vq, scale, see)
            if self.dtype == "bf16":
                # the result's rounding; the probabilities' to fp16, 2^-11 of each, and as much for scores, sums and exponentials
                tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * reach
            else:
                # queries and probabilities to 22 bits, exponentials and sums to fp32; a score is off by that much of its terms
                tol = 2.0 ** -20 * reach * (1.0 + big[..., None])
            d = np.abs(got[b] - want)
            assert np.all(d <= tol + 1e-30), (b, L, float((d / (tol + 1e-30)).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,Hkv,G", [(64, 4, 1), (128, 2, 1), (128, 1, 7), (64, 1, 8), (128, 1, 5), (64, 2, 3)])
@pytest.mark.parametrize("n_q", [1, 3, 8])
def test_attention_over_uneven_sequences(dtype, dh, Hkv, G, n_q):
    f = Filled(dtype, dh, Hkv, G, [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, 130, 511], n_q, seed=dh + G + n_q)
    f.put()
    f.check(f.cache.attention(f.q, f.rows, n_q=n_q))


@pytest.mark.parametrize("dtype,dh,Hkv,G,n_q", [("bf16", 128, 2, 7, 17), ("bf16", 64, 1, 8, 61), ("f32", 128, 1, 1, 33), ("bf16", 128, 1, 16, 5),
                                                ("f32", 64, 1, 40, 2)])
def test_attention_with_many_columns(dtype, dh, Hkv, G, n_q):
    f = Filled(dtype, dh, Hkv, G, [700, 5, 64], n_q, seed=3)
    f.put()
    f.check(f.cache.attention(f.q, f.rows, n_q=n_q))


def _words(mask):
    t = _torch()
    B, n_q, T = mask.shape
    w = (T + 31) // 32
    bits = np.zeros((B, n_q, w * 32), np.uint32)
    bits[..., :T] = mask
    return t.from_numpy((bits.reshape(B, n_q, w, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32).view(np.int32)).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,mask_rows,lens", [(1, 1, [1, 40]), (5, 5, [5, 3, 200]), (10, 51, [60, 51, 20, 333]), (61, 61, [61, 100, 10]),
                                                (16, 241, [300, 241, 240]), (3, 1024, [40, 1100])])
def test_attention_under_a_tree_mask(dtype, n_q, mask_rows, lens):
    f = Filled(dtype, 128, 2, 2, lens, n_q, seed=n_q)
    f.put()
    mask = f.rng.random((len(lens), n_q, mask_rows)) < 0.4
    mask[:, 0] = False                                               # a query that sees nothing of the last rows
    mask[0, -1] = True
    f.check(f.cache.attention(f.q, f.rows, n_q=n_q, mask=_words(mask), mask_rows=mask_rows), mask, mask_rows)


@pytest.mark.parametrize("fill", [0xFF, 0x7F, 0x00])
def test_what_lies_behind_the_rows_does_not_matter(fill):
    """Rows that were never written (NaN, infinite and zero parameters), and rows that a query does not see, holding NaN."""
    t = _torch()
    f = Filled("bf16", 128, 2, 3, [1, 18, 47, 80], 4, seed=11, fill=fill, max_len=96)
    f.put()
    out = f.cache.attention(f.q, f.rows, n_q=4)
    f.check(out)
    # the sequence's last row is NaN: only the last query sees it
    cu = _starts(f.lens)
    bad = t.full((4, 2, 128), math.nan, dtype=t.bfloat16, device="cuda")
    f.cache.append(bad, bad, [0, 1, 2, 3, 4], _ints([n - 1 for n in f.lens]))
    again = f.cache.attention(f.q, f.rows, n_q=4).view(4, 4, 6, 128)
    out = out.view(4, 4, 6, 128)
    assert t.equal(again[:, :3], out[:, :3])
    assert bool(again[:, 3].isnan().all())
    assert cu[-1] == 146


def test_infinite_rows_that_are_masked_by_a_tree():
    t = _torch()
    f = Filled("bf16", 64, 1, 8, [70], 2, seed=12)
    f.v[66] = math.inf
    f.k[67] = math.nan
    f.put()
    mask = np.ones((1, 2, 10), bool)
    mask[0, :, 6] = mask[0, :, 7] = False                            # rows 66 and 67
    out = f.cache.attention(f.q, f.rows, n_q=2, mask=_words(mask), mask_rows=10)
    f.k[67], f.v[66] = 0.0, 0.0
    f.check(out, mask, 10)
    assert bool(t.isfinite(out).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_and_values_of_any_size(dtype):
    """Queries from 2^-60 to flat-out certain, values whose rows differ by factors of a thousand."""
    for q_std, spread in ((2.0 ** -60, 0.0), (30.0, 0.0), (1.0, 3.5), (8.0, 3.5)):
        f = Filled(dtype, 128, 1, 4, [257, 40], 2, seed=13, q_std=q_std, spread=spread)
        f.put()
        f.check(f.cache.attention(f.q, f.rows, n_q=2))


@pytest.mark.parametrize("scale_v", [1e-30, 1e-6, 1e6, 1e30])
def test_values_of_any_magnitude(scale_v):
    f = Filled("bf16", 128, 1, 1, [300], 1, seed=14)
    f.v *= scale_v
    f.put()
    f.check(f.cache.attention(f.q, f.rows))


def test_scores_that_keep_rising():
    """Every row beats all before it by a little: the maximum is raised late, and often."""
    t = _torch()
    for slope in (0.02, 0.5, 3.0):
        f = Filled("bf16", 64, 1, 1, [900], 1, seed=15)
        d = t.nn.functional.normalize(f.q[0, 0].float(), dim=0)
        f.k[:, 0] = (f.k[:, 0].float() * 0.1 + t.arange(900, device="cuda")[:, None] * slope * 8.0 / float(f.q[0, 0].float().norm()) * d).bfloat16()
        f.put()
        f.check(f.cache.attention(f.q, f.rows))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_slots_and_an_output_of_the_callers(dtype):
    t = _torch()
    f = Filled(dtype, 64, 2, 4, [100, 37, 5], 2, seed=16, slots=[5, 0, 3], max_len=160)
    f.put()
    wide = t.zeros((6, 1024), dtype=f.q.dtype, device="cuda")
    wide[:, 256:768] = f.q.reshape(6, 512)
    out = t.full((6, 640), 7.0, dtype=f.q.dtype, device="cuda")
    got = f.cache.attention(wide[:, 256:768].view(6, 8, 64), f.rows, n_q=2, slots=[5, 0, 3], out=out[:, :512].view(6, 8, 64))
    f.check(got)
    assert bool((out[:, 512:] == 7.0).all())


@pytest.mark.parametrize("B,Hkv,G,dh,lens", [(1, 1, 8, 64, [20001]), (2, 4, 7, 128, [9000, 4097]), (64, 1, 1, 64, list(range(1, 65)))])
def test_long_and_many(B, Hkv, G, dh, lens):
    f = Filled("bf16", dh, Hkv, G, lens, 1, seed=17)
    f.put()
    f.check(f.cache.attention(f.q, f.rows))


def test_row_counts_outside_the_cache_are_read_as_its_ends():
    t = _torch()
    f = Filled("bf16", 128, 1, 2, [64, 64], 1, seed=18, max_len=64)
    f.put()
    out = f.cache.attention(f.q, _ints([-5, 1000]))
    whole = f.cache.attention(f.q, _ints([64, 64]))
    assert bool((out[0] == 0).all()) and t.equal(out[1], whole[1])


def test_the_same_call_gives_the_same_bits():
    t = _torch()
    f = Filled("bf16", 128, 4, 7, [3000, 777], 3, seed=19)
    f.put()
    first = f.cache.attention(f.q, f.rows, n_q=3)
    for _ in range(5):
        assert t.equal(f.cache.attention(f.q, f.rows, n_q=3), first)


def test_a_cache_of_more_than_four_gigabytes():
    t = _torch()
    cache = _cache(40, 32, 128, 65536)                               # 5.4 GB of codes for the keys alone
    rng = np.random.default_rng(20)
    k, v = (_to(rng.standard_normal((50, 32, 128)), "bf16") for _ in range(2))
    q = _to(rng.standard_normal((1, 32, 128)), "bf16")
    small = _cache(1, 32, 128, 65536)
    cache.append(k, v, [0, 50], _ints([0]), [39])
    small.append(k, v, [0, 50], _ints([0]))
    assert t.equal(cache.attention(q, _ints([50]), slots=[39]), small.attention(q, _ints([50])))
    cache.append(k, v, [0, 50], _ints([65536 - 50]), [38])
    got, _ = cache.read([0, 50], _ints([65536 - 50]), [38])
    want, _ = small.read([0, 50], _ints([0]))
    assert t.equal(got, want)


def test_captured_calls_replay_with_new_inputs():
    t = _torch()
    f = Filled("bf16", 128, 2, 4, [50, 90], 1, seed=21, max_len=128)
    f.put()
    out = t.empty_like(f.q)
    k_new, v_new, start = f.k[:2].clone(), f.v[:2].clone(), _ints([50, 90])
    rows = _ints([51, 91])

    def step():
        f.cache.append(k_new, v_new, [0, 1, 2], start)
        f.cache.attention(f.q, rows, out=out)

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        step()
    t.cuda.current_stream().wait_stream(side)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        step()
    for i in range(3):
        k_new.copy_(f.k[2 + 2 * i:4 + 2 * i])
        v_new.copy_(f.v[2 + 2 * i:4 + 2 * i])
        graph.replay()
        got = out.clone()
        step()
        assert t.equal(got, out)
        start += 1
        rows += 1


def test_two_streams_at_once():
    t = _torch()
    f = Filled("bf16", 128, 4, 2, [2000, 1500], 2, seed=22)
    f.put()
    want = f.cache.attention(f.q, f.rows, n_q=2)
    streams = [t.cuda.Stream() for _ in range(2)]
    got = []
    t.cuda.synchronize()
    for i in range(20):
        with t.cuda.stream(streams[i % 2]):
            got.append(f.cache.attention(f.q, f.rows, n_q=2))
    t.cuda.synchronize()
    assert all(t.equal(g, want) for g in got)


def test_tensors_that_do_not_fit_are_refused():
    t = _torch()
    cache = _cache(2, 2, 64, 32)
    k = t.zeros((4, 2, 64), dtype=t.bfloat16, device="cuda")
    q = t.zeros((2, 4, 64), dtype=t.bfloat16, device="cuda")
    rows = _ints([3, 3])
    for call in (lambda: cache.append(k, k.float(), [0, 4], _ints([0])), lambda: cache.append(k, k, [0, 3], _ints([0])),
                 lambda: cache.append(k.transpose(1, 2), k.transpose(1, 2), [0, 4], _ints([0])),
                 lambda: cache.append(k, k, [0, 4], _ints([0, 0])), lambda: cache.append(k.cpu(), k, [0, 4], _ints([0])),
                 lambda: cache.attention(q, rows.long()), lambda: cache.attention(q[:1], rows), lambda: cache.attention(q, rows, n_q=2),
                 lambda: cache.attention(q, rows, mask=t.zeros((2, 1, 1), dtype=t.int32, device="cuda"), mask_rows=33),
                 lambda: cache.attention(q, rows, out=t.zeros((2, 4, 64), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        cache.append(k.half(), k.half(), [0, 4], _ints([0]))
    for bad in ((0, 2, 64, 32), (1, 0, 64, 32), (1, 2, 96, 32), (1, 2, 64, 0)):
        with pytest.raises(ValueError):
            _cache(*bad)


@pytest.mark.parametrize("call", ["append", "attention", "logprobs"])
def test_a_first_call_may_be_a_captured_one(call):
    """In a process of its own: nothing has been loaded or set up when the capture begins."""
    import subprocess
    import sys
    code = f"""
import torch
from paper_2509_23928_b200 import Kv4Cache, logprobs
cache = Kv4Cache(2, 2, 64, 64)
k = torch.randn(10, 2, 64, device="cuda").bfloat16()
q = torch.randn(2, 4, 64, device="cuda").bfloat16()
x = torch.randn(3, 500, device="cuda")
zero, rows = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([5, 5], dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
f = dict(append=lambda: cache.append(k, k, [0, 5, 10], zero), attention=lambda: cache.attention(q, rows), logprobs=lambda: logprobs(x, top_n=3))["{call}"]
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    out = f()
g.replay()
torch.cuda.synchronize()
got = cache.data.clone() if out is None else out.clone() if torch.is_tensor(out) else out.top_logprobs.clone()
again = f()
assert torch.equal(got, cache.data if again is None else again if torch.is_tensor(again) else again.top_logprobs)
print("done")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stderr[-2000:]


def test_the_output_may_be_the_queries():
    t = _torch()
    for n_q, G in ((1, 2), (5, 7)):
        f = Filled("bf16", 128, 2, G, [1500, 33], n_q, seed=23)
        f.put()
        want = f.cache.attention(f.q, f.rows, n_q=n_q)
        q = f.q.clone()
        assert t.equal(f.cache.attention(q, f.rows, n_q=n_q, out=q), want) and t.equal(q, want)


# ---------------------------------------------------------------- many columns of bf16 queries (blocks of 64, 128 rows at a time)
def _check_many(f, out, mask=None, mask_rows=0):
    """Filled.check, and a score's error: its row's values are rounded to 11 bits, each by at most 2^-11 of itself.  As independent errors
    of rms 2^-11 / sqrt(3) they add up to 6 * 2^-11 / sqrt(3) < 2^-9 of the root of the sum of the products' squares, six sigma; a weight,
    and the sum that it is divided by, are off by as much."""
    cu = _starts(f.lens)
    got, q = _np(out).reshape(len(f.lens), f.n_q, f.Hkv * f.G, f.dh), _np(f.q).reshape(len(f.lens), f.n_q, -1, f.dh)
    scale = f.dh ** -0.5
    for b, L in enumerate(f.lens):
        kq, vq = ref.quantise(_np(f.k[cu[b]:cu[b + 1]])), ref.quantise(_np(f.v[cu[b]:cu[b + 1]]))
        see = ref.visible(L, f.n_q, None if mask is None else mask[b], mask_rows)
        want, reach, _ = ref.attention(q[b], kq, vq, scale, see)
        ds = np.zeros((f.n_q, f.Hkv * f.G, 1))
        if L:
            kk = np.repeat(ref.values(*kq), f.G, axis=1)
            ds = 2.0 ** -9 * scale * np.sqrt(np.einsum("qhd,lhd->qhl", q[b] ** 2, kk ** 2)).max(-1, keepdims=True)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.0 * np.expm1(ds)) * reach
        d = np.abs(got[b] - want)
        assert np.all(d <= tol + 1e-30), (b, L, float((d / (tol + 1e-30)).max()))


@pytest.mark.parametrize("dh,Hkv,G,n_q", [(128, 2, 1, 17), (128, 1, 7, 8), (128, 1, 1, 64), (128, 1, 5, 64), (64, 1, 7, 7), (64, 2, 1, 64), (64, 1, 8, 33)])
def test_many_columns_over_uneven_sequences(dh, Hkv, G, n_q):
    f = Filled("bf16", dh, Hkv, G, [0, 1, 2, 15, 17, 63, 64, 65, 127, 128, 129, 200, 255, 257, 640, 1030], n_q, seed=dh + G + n_q)
    f.put()
    _check_many(f, f.cache.attention(f.q, f.rows, n_q=n_q))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("max_len", [1024, 32768])
@pytest.mark.parametrize("rising", [True, False])
def test_many_columns_whose_scores_rise_and_fall(dh, max_len, rising):
    """The running maximum and the values' scale change from step to step; max_len says how many CTAs share a sequence."""
    t = _torch()
    f = Filled("bf16", dh, 2, 1, [1024, 900, 385], 56, seed=31, max_len=max_len)
    d = t.nn.functional.normalize(f.q[:56, 0].float().mean(0), dim=0)
    cu = _starts(f.lens)
    for b, n in enumerate(f.lens):
        r = t.arange(n, device="cuda").float()
        slope = r if rising else n - r
        f.k[cu[b]:cu[b + 1]] = (f.k[cu[b]:cu[b + 1]].float() * 0.1 + (slope * 0.2)[:, None, None] * d).bfloat16()
        f.v[cu[b]:cu[b + 1]] *= (10.0 ** ((r // 128) % 5 - 2))[:, None, None].bfloat16()
    f.put()
    _check_many(f, f.cache.attention(f.q, f.rows, n_q=56))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("fill", [0xFF, 0x7F, 0x00])
def test_many_columns_take_nothing_of_rows_they_do_not_see(dh, fill):
    t = _torch()
    f = Filled("bf16", dh, 1, 1, [0, 1, 60, 61, 127, 130, 300], 61, seed=37, fill=fill)
    f.put()
    _check_many(f, f.cache.attention(f.q, f.rows, n_q=61))
    # a group of a row of values is NaN: those channels of the queries that see it, nothing else
    for r in (0, 40, 255, 299):
        f = Filled("bf16", dh, 1, 1, [300], 61, seed=41)
        f.put()
        clean = f.cache.attention(f.q, f.rows, n_q=61).reshape(61, dh)
        f.v[r, 0, 32:] = math.nan
        f.put()
        out = f.cache.attention(f.q, f.rows, n_q=61).reshape(61, dh)
        sees = t.arange(61, device="cuda") + 300 - 61 >= r
        assert bool(out[sees][:, 32:].isnan().all()) and not bool(out[~sees].isnan().any()) and not bool(out[:, :32].isnan().any()), r
        assert t.equal(out[~sees], clean[~sees])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("mask_rows,lens", [(61, [61, 100, 10, 300]), (333, [333, 400, 20, 129]), (1024, [1000, 1024, 1, 0])])
def test_many_columns_under_a_mask(dh, mask_rows, lens):
    f = Filled("bf16", dh, 2, 1, lens, 61, seed=mask_rows)
    f.put()
    mask = f.rng.random((4, 61, mask_rows)) < 0.4
    mask[:, 3] = False
    mask[1, 5:9, : mask_rows // 2] = False
    _check_many(f, f.cache.attention(f.q, f.rows, n_q=61, mask=_words(mask), mask_rows=mask_rows), mask, mask_rows)


@pytest.mark.parametrize("scale_v", [1e-30, 1e-6, 1e6, 1e30, 1e37])
@pytest.mark.parametrize("dh", [64, 128])
def test_many_columns_of_values_of_any_magnitude(dh, scale_v):
    f = Filled("bf16", dh, 1, 1, [300], 61, seed=43)
    f.v *= scale_v
    f.put()
    _check_many(f, f.cache.attention(f.q, f.rows, n_q=61))


def test_many_columns_of_queries_of_any_size():
    for q_std, spread in ((2.0 ** -60, 0.0), (30.0, 0.0), (1.0, 3.5), (8.0, 3.5)):
        f = Filled("bf16", 128, 1, 4, [257, 40], 9, seed=44, q_std=q_std, spread=spread)
        f.put()
        _check_many(f, f.cache.attention(f.q, f.rows, n_q=9))


def test_many_columns_of_strided_queries_and_outputs():
    t = _torch()
    f = Filled("bf16", 128, 2, 2, [500, 77], 20, seed=47)
    f.put()
    want = f.cache.attention(f.q, f.rows, n_q=20)
    wide = t.full((40, 1024), 7.0, dtype=t.bfloat16, device="cuda")
    wide[:, 256:768] = f.q.reshape(40, 512)
    out = t.full((40, 1536), 3.0, dtype=t.bfloat16, device="cuda")
    f.cache.attention(wide[:, 256:768].view(40, 4, 128), f.rows, n_q=20, out=out[:, 512:1024].view(40, 4, 128))
    assert t.equal(out[:, 512:1024], want.reshape(40, 512))
    assert bool((out[:, :512] == 3).all()) and bool((out[:, 1024:] == 3).all())
    for _ in range(5):
        assert t.equal(f.cache.attention(f.q, f.rows, n_q=20), want)


def test_many_columns_on_two_streams_and_in_graphs():
    """Calls that overlap on the GPU share nothing; a replayed call reads the lengths, queries and rows of its replay."""
    t = _torch()
    fs = [Filled("bf16", dh, 2, 1, [900, 31, 400], 61, seed=50 + dh) for dh in (64, 128)]
    want = []
    for f in fs:
        f.put()
        want.append(f.cache.attention(f.q, f.rows, n_q=61).clone())
    graphs, outs, streams = [], [], [t.cuda.Stream(), t.cuda.Stream()]
    for f, s in zip(fs, streams):
        s.wait_stream(t.cuda.current_stream())
        out = t.zeros_like(f.q)
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g, stream=s):
            for _ in range(3):
                f.cache.attention(f.q, f.rows, n_q=61, out=out)
        graphs.append(g)
        outs.append(out)
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with t.cuda.stream(s):
                g.replay()
    t.cuda.synchronize()
    for o, w in zip(outs, want):
        assert t.equal(o, w)
    for f, g, o in zip(fs, graphs, outs):
        f.lens = [123, 1, 0]
        f.rows.copy_(_ints(f.lens))
        f.q.mul_(0.5)
        g.replay()
        t.cuda.synchronize()
        assert t.equal(o, f.cache.attention(f.q, f.rows, n_q=61))
        assert bool((o.view(3, 61, -1)[2] == 0).all()) and bool((o.view(3, 61, -1)[1, :60] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["halves", "eighths", "spread", "tiny beside large", "nearly ties"])
def test_codes_of_values_beside_ties(dtype, kind):
    """Half a million values of which many are ties, or a last bit away from one: the codes are those of exact arithmetic."""
    t = _torch()
    g = t.Generator(device="cuda").manual_seed(7)
    shape = (1024, 4, 128)
    x = t.randn(shape, device="cuda", generator=g)
    if kind == "halves":
        x = t.randint(0, 31, shape, device="cuda", generator=g).float() * 0.5
    elif kind == "eighths":
        x = (x * 8).round() / 8
    elif kind == "spread":
        x = x * t.exp2(t.randint(-20, 20, shape, device="cuda", generator=g).float())
    elif kind == "tiny beside large":
        x = t.where(t.rand(shape, device="cuda", generator=g) < 0.5, x * 1e-6, x)
    else:
        x = t.randint(-60, 61, shape, device="cuda", generator=g).float() * 2.0 ** -3 + x * 2.0 ** -14 * (t.rand(shape, device="cuda", generator=g) < 0.3)
    x = x.to(t.bfloat16 if dtype == "bf16" else t.float32)
    cache = _cache(1, 4, 128, 1024)
    cache.append(x, x, [0, 1024], _ints([0]))
    k, v = cache.read([0, 1024], _ints([0]))
    want = ref.values(*ref.quantise(_np(x))).astype(np.float32)
    assert np.array_equal(k.cpu().numpy(), want) and np.array_equal(v.cpu().numpy(), want)


@pytest.mark.parametrize("n_q", [1, 33])
def test_counts_and_masks_that_start_anywhere(n_q):
    t = _torch()
    f = Filled("bf16", 128, 2, 2, [70, 33, 100], n_q, seed=61)
    f.put()
    again = _cache(3, 2, 128, 100)
    zeros = t.zeros(5, dtype=t.int32, device="cuda")
    again.append(f.k, f.v, _starts(f.lens), zeros[1:4])
    for a, b in zip(again.read([0, 70, 103, 203], zeros[2:]), f.cache.read([0, 70, 103, 203], _ints([0, 0, 0]))):
        assert t.equal(a, b)
    wide = _ints([7] + f.lens)
    assert t.equal(again.attention(f.q, wide[1:], n_q=n_q), f.cache.attention(f.q, f.rows, n_q=n_q))
    mask = f.rng.random((3, n_q, 40)) < 0.5
    words = t.zeros(1 + 3 * n_q * 2, dtype=t.int32, device="cuda")
    words[1:] = _words(mask).view(-1)
    out = again.attention(f.q, wide[1:], n_q=n_q, mask=words[1:].view(3, n_q, 2), mask_rows=40)
    assert t.equal(out, f.cache.attention(f.q, f.rows, n_q=n_q, mask=_words(mask), mask_rows=40))


def _check_weights(f, out, see):
    """Results whose weights are the same for every row of see [sequence][n_q, rows]: the values' share of Filled.check's bounds alone."""
    got, cu = _np(out).reshape(len(f.lens), f.n_q, f.Hkv * f.G, f.dh), _starts(f.lens)
    for b, n in enumerate(f.lens):
        kq, vq = ref.quantise(_np(f.k[cu[b]:cu[b + 1]])), ref.quantise(_np(f.v[cu[b]:cu[b + 1]]))
        want, reach, _ = ref.attention(np.zeros((f.n_q, f.Hkv * f.G, f.dh)), kq, vq, 1.0, see[b])
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * reach if f.dtype == "bf16" else 2.0 ** -20 * reach
        d = np.abs(got[b] - want)
        assert np.all(d <= tol), (b, float((d / np.maximum(tol, 1e-300)).max()))


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("bf16", 61), ("f32", 1), ("f32", 20)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("size,sign", [(1e3, 1), (1e5, -1), (1e5, 1), (1e8, 1), (1e12, -1), (1e16, -1), (1e18, -1), (1e18, 1)])
def test_scores_far_from_zero(dtype, n_q, dh, size, sign):
    """Scores of 1e7 to 1e37 are scores like any other: equal ones share the weight; one that is half as high has none, or all if they are below zero."""
    f = Filled(dtype, dh, 2, 1, [300, 3], n_q, seed=63)
    f.q.fill_(1.37 * size)
    f.k.fill_(sign * 1.71 * size)
    f.put()
    see = [ref.visible(n, n_q, None, 0) for n in f.lens]
    _check_weights(f, f.cache.attention(f.q, f.rows, n_q=n_q), see)
    for b, r in ((0, 280), (1, 1)):
        f.k[_starts(f.lens)[b] + r] *= 0.5
        s, other = see[b], np.arange(f.lens[b]) != r
        if sign < 0:
            s[s[:, r]] = ~other
        else:
            s[s[:, other].any(-1), r] = False
    f.put()
    _check_weights(f, f.cache.attention(f.q, f.rows, n_q=n_q), see)


@pytest.mark.parametrize("dtype,n_q", [("bf16", 4), ("bf16", 61), ("f32", 4), ("f32", 20)])
@pytest.mark.parametrize("dh", [64, 128])
def test_scales_that_are_tiny_or_huge(dtype, n_q, dh):
    """Queries and a scale so small that all scores are next to 0, rows that are not seen among them; and so large that only a 0 is one."""
    f = Filled(dtype, dh, 2, 1, [300, 3, 70], n_q, seed=65)
    f.q *= 1e-30
    f.put()
    see = [ref.visible(n, n_q, None, 0) for n in f.lens]
    _check_weights(f, f.cache.attention(f.q, f.rows, n_q=n_q, scale=1e-20), see)
    f.q *= 1e30
    f.q *= 1e30
    f.k.zero_()
    f.put()
    _check_weights(f, f.cache.attention(f.q, f.rows, n_q=n_q, scale=9e37), see)


@pytest.mark.parametrize("dtype,n_q", [("bf16", 1), ("f32", 1), ("bf16", 2)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("scale_v", [1e33, 1e34, 5e34])
def test_values_next_to_the_end_of_the_range(dtype, n_q, dh, scale_v):
    """2^8 |v| summed over the rows stays below 2^127: so far values are taken."""
    f = Filled(dtype, dh, 1, 1, [3, 1], n_q, seed=67)
    f.v.clamp_(-4.0, 4.0).mul_(scale_v)
    assert 256.0 * 3 * 4.0 * scale_v < 2.0 ** 127
    f.k.zero_()
    f.put()
    _check_weights(f, f.cache.attention(f.q, f.rows, n_q=n_q), [ref.visible(n, n_q, None, 0) for n in f.lens])


def _unseen(f, size, hidden):
    """Rows `hidden` [sequence][...] of f with keys and values of about `size`, or zeros."""
    g = _torch().Generator(device="cuda").manual_seed(5)
    for b, rows in enumerate(hidden):
        i = [_starts(f.lens)[b] + r for r in rows]
        for x in (f.k, f.v):
            x[i] = (x[i].float().normal_(0.0, 1.0, generator=g) * size).to(x.dtype)
    f.put()


UNSEEN = [("bf16", 64, 1, 4), ("bf16", 128, 1, 4), ("bf16", 128, 2, 5), ("f32", 64, 1, 4), ("f32", 128, 3, 6),
          ("bf16", 128, 1, 33), ("bf16", 64, 2, 33), ("bf16", 128, 7, 8)]


def _check_any(f, out, mask=None, mask_rows=0):
    many = f.dtype == "bf16" and f.G * f.n_q > (16 if f.dh == 128 else 48)
    _check_many(f, out, mask, mask_rows) if many else f.check(out, mask, mask_rows)


@pytest.mark.parametrize("dtype,dh,G,n_q", UNSEEN)
@pytest.mark.parametrize("size", [1e4, 1e8, 1e12, 1e30, 1e-20])
def test_rows_that_are_not_seen_may_hold_anything(dtype, dh, G, n_q, size):
    """Finite rows far larger (or smaller) than the others, hidden from all queries by a mask, from some, and by the causal edge: to the bit what
    the same call gives where those rows are zero, and within the bounds."""
    t = _torch()
    lens, T = [300, 70, 45], 40
    f = Filled(dtype, dh, 2, G, lens, n_q, seed=71)
    mask = f.rng.random((3, n_q, T)) < 0.6
    everywhere, half = [3, 4, 17, 30], [8, 20, 33]                   # of the last T rows: hidden from all, from the first queries
    mask[:, :, everywhere] = False
    mask[:, :n_q // 2, half] = False
    mask[:, n_q // 2:, half] = True
    got = []
    for s in (0.0, size):
        _unseen(f, s, [[n - T + j for j in everywhere + half] for n in lens])
        got.append(f.cache.attention(f.q, f.rows, n_q=n_q, mask=_words(mask), mask_rows=T).view(3, n_q, -1))
        if s == 0.0:
            _check_any(f, got[0], mask, T)
    assert bool(t.isfinite(got[1]).all())
    assert t.equal(got[0][:, :n_q // 2], got[1][:, :n_q // 2])
    got = []
    for s in (0.0, size):
        _unseen(f, s, [[n - 1] for n in lens])                       # the last query alone sees it
        got.append(f.cache.attention(f.q, f.rows, n_q=n_q).view(3, n_q, -1))
    assert bool(t.isfinite(got[1]).all())
    assert t.equal(got[0][:, :n_q - 1], got[1][:, :n_q - 1])


@pytest.mark.parametrize("dtype,dh,G,n_q", UNSEEN)
@pytest.mark.parametrize("fill", [0xFF, 0xFE, 0x7F, 0x7E, 0x80, "random"])
def test_rows_that_were_never_written_may_be_masked(dtype, dh, G, n_q, fill):
    """A padded tree over a buffer with anything in it: the mask leaves the padding out."""
    t = _torch()
    f = Filled(dtype, dh, 2, G, [40, 21], n_q, seed=73, max_len=96)
    mask = np.zeros((2, n_q, 64), bool)
    want = None
    for b, n in enumerate(f.lens):
        mask[b, :, :n] = f.rng.random((n_q, n)) < 0.7                # the rows [rows - 64, rows) = [0, 64): n of them written
    rows = _ints([64, 64])
    outs = []
    for what in (0, fill):
        if what == "random":
            g = t.Generator(device="cuda").manual_seed(9)
            f.cache.data.random_(0, 256, generator=g)
        else:
            f.cache.data.fill_(what)
        f.put()
        outs.append(f.cache.attention(f.q, rows, n_q=n_q, mask=_words(mask), mask_rows=64))
    assert bool(t.isfinite(outs[0]).all()) and t.equal(outs[0], outs[1])


@pytest.mark.parametrize("dtype,dh,G,n_q", UNSEEN)
@pytest.mark.parametrize("size", [1e4, 1e12, 1e30])
@pytest.mark.parametrize("first", [True, False])
def test_rows_that_are_seen_without_weight_take_no_bits(dtype, dh, G, n_q, size, first):
    """A far larger row whose score is 400 below the others (their scores: within 200): seen before them, or after."""
    f = Filled(dtype, dh, 1, G, [400, 80], n_q, seed=75)
    f.q.copy_(f.q.abs() + 0.5)
    f.k.copy_((f.k.float() * 0.05).to(f.k.dtype))
    cu = _starts(f.lens)
    got = []
    for s in (0.0, size):
        for b in range(2):
            i = slice(cu[b], cu[b] + 3) if first else slice(cu[b + 1] - n_q - 3, cu[b + 1] - n_q)
            f.k[i] = -400.0
            f.v[i] = (f.v[i].float().sign() * s).to(f.v.dtype)
        f.put()
        got.append(f.cache.attention(f.q, f.rows, n_q=n_q))
        f.v[:] = f.v.where(f.v != 0, 1.0)
    assert _torch().equal(got[0], got[1])


@pytest.mark.parametrize("dtype,dh,G,n_q", UNSEEN)
def test_groups_of_channels_of_other_magnitudes(dtype, dh, G, n_q):
    """Neighbouring groups of 32 channels whose values differ by 1e4: every channel has the precision of its own group."""
    f = Filled(dtype, dh, 2, G, [300, 20], n_q, seed=77)
    f.v[:, :, 32:64] *= 1e-4
    f.q *= 0.3
    f.put()
    _check_any(f, f.cache.attention(f.q, f.rows, n_q=n_q))


@pytest.mark.parametrize("dtype,dh,G,n_q", UNSEEN)
@pytest.mark.parametrize("step", [2.0 ** 10, 2.0 ** -10, 2.0 ** 25, 2.0 ** -25])
@pytest.mark.parametrize("rising", [True, False])
def test_values_and_scores_that_change_together(dtype, dh, G, n_q, step, rising):
    """Values that grow (or shrink) by `step` every 70 rows while scores rise (or fall): every query's largest weight x value is somewhere else."""
    t = _torch()
    f = Filled(dtype, dh, 1, G, [600, 90], n_q, seed=79, max_len=4096)
    f.q.copy_(f.q.abs() * 0.25)
    for b in range(2):
        i = slice(_starts(f.lens)[b], _starts(f.lens)[b + 1])
        r = t.arange(f.lens[b], device="cuda")[:, None, None]
        f.k[i] = (f.k[i].float() * 0.02 + (r if rising else 600 - r) * 0.03).to(f.k.dtype)
        f.v[i] = (f.v[i].double() * step ** (r // 70 % 4).double()).to(f.v.dtype)
    f.put()
    _check_any(f, f.cache.attention(f.q, f.rows, n_q=n_q))


@pytest.mark.parametrize("dh,G,n_q", [(64, 1, 1), (128, 1, 1), (64, 4, 5), (128, 2, 8)])
@pytest.mark.parametrize("ratio", [1e-2, 1e-4, 1e-5])
def test_fp32_weights_keep_22_bits_in_every_group(dh, G, n_q, ratio):
    """A group of channels far smaller than its neighbour, few rows with scores around 0: the bounds of its own values."""
    f = Filled("f32", dh, 2, G, [3, 40, 2, 20], n_q, seed=81)
    f.v[:, :, 32:64] *= ratio
    f.k *= 0.1
    f.put()
    f.check(f.cache.attention(f.q, f.rows, n_q=n_q))


@pytest.mark.parametrize("dtype,dh,G,n_q", UNSEEN)
@pytest.mark.parametrize("at", [0, 130, 299])
def test_a_row_of_zeros_that_takes_the_weight(dtype, dh, G, n_q, at):
    """Where a row without values has all the weight but 1e-12, what the others add to its zeros is held like any result."""
    f = Filled(dtype, dh, 2, G, [300, 100], n_q, seed=83, q_std=0.5)
    f.q.copy_(f.q.abs() + 0.1)
    f.k.copy_((f.k.float() * 0.1).to(f.k.dtype))
    for b in range(2):
        r = _starts(f.lens)[b] + min(at, f.lens[b] - n_q)
        f.v[r] = 0.0
        f.k[r] = 60.0 / (float(f.q.float().mean()) * dh ** 0.5)
    f.put()
    _check_any(f, f.cache.attention(f.q, f.rows, n_q=n_q))


@pytest.mark.parametrize("mask_rows", [0, -1])
def test_a_mask_of_no_rows_is_refused(mask_rows):
    """An empty tensor has no address: without the refusal the call would be a causal one."""
    t = _torch()
    f = Filled("bf16", 64, 1, 2, [20, 20], 3, seed=85)
    f.put()
    with pytest.raises(ValueError, match="mask_rows"):
        f.cache.attention(f.q, f.rows, n_q=3, mask=t.zeros((2, 3, 0), dtype=t.int32, device="cuda"), mask_rows=mask_rows)
