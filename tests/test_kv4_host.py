"""What the context-free calls on a 4-bit cache refuse before anything is launched (no GPU is touched)."""
import ctypes as C

import pytest

P = 0x10000                      # an address that is aligned and never read


def _cache(**kw):
    from paper_2509_23928_b200.binding import hivis_kv4_cache
    base = dict(struct_size=C.sizeof(hivis_kv4_cache), n_slots=4, n_kv_heads=2, head_dim=64, max_len=64, data=P)
    base.update(kw)
    return hivis_kv4_cache(**base)


def _ints(x):
    return None if x is None else (C.c_int * len(x))(*x)


def _append(cache, B=2, slots=None, cu=(0, 1, 3), start=P, k=P, v=P, dtype=1, ld=128):
    from paper_2509_23928_b200.binding import lib
    return lib.hivis_kv4_append(None if cache is None else C.byref(cache), B, _ints(slots), _ints(cu), start, k, v, dtype, ld, None)


def _read(cache, B=2, slots=None, cu=(0, 1, 3), start=P, k=P, v=P):
    from paper_2509_23928_b200.binding import lib
    return lib.hivis_kv4_read(None if cache is None else C.byref(cache), B, _ints(slots), _ints(cu), start, k, v, None)


def _attend(cache, B=2, slots=None, rows=P, n_q=1, heads=4, q=P, dtype=1, q_ld=256, scale=0.125, mask=None, mask_rows=0, out=P, out_ld=256):
    from paper_2509_23928_b200.binding import lib
    return lib.hivis_kv4_attention(None if cache is None else C.byref(cache), B, _ints(slots), rows, n_q, heads, q, dtype, q_ld, scale,
                                   mask, mask_rows, out, out_ld, None)


@pytest.mark.parametrize("kw,code", [
    (dict(struct_size=8), -1), (dict(head_dim=96), -2), (dict(head_dim=32), -2), (dict(n_kv_heads=0), -2), (dict(n_slots=0), -2),
    (dict(max_len=0), -2), (dict(max_len=33), -2), (dict(max_len=2 ** 28 + 32), -2), (dict(data=None), -1),
    (dict(data=P + 8), -1), (dict(n_kv_heads=70000), -2),
])
def test_a_bad_cache_is_refused_by_every_call(kw, code):
    from paper_2509_23928_b200 import hivis_last_error
    for call in (_append, _read, _attend):
        assert call(_cache(**kw)) == code
        assert "hivis_kv4" in hivis_last_error(None)
    assert _append(None) == _read(None) == _attend(None) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -5), (dict(B=65), -5), (dict(slots=(0, 4)), -1), (dict(slots=(1, -1)), -1), (dict(slots=(3, 3)), -1),
    (dict(cu=(1, 1, 3)), -1), (dict(cu=(0, 3, 1)), -1), (dict(cu=(0, 65, 66)), -5), (dict(start=None), -1), (dict(start=P + 4), -1),
    (dict(cu=(0, -2147483648, 2147483647)), -1), (dict(k=None), -1), (dict(v=P + 2), -1),
])
def test_bad_rows_are_refused(kw, code):
    assert _append(_cache(), **kw) == code
    assert _read(_cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -3), (dict(ld=120), -2), (dict(ld=132), -2), (dict(ld=0), -2)])
def test_bad_inputs_of_append_are_refused(kw, code):
    assert _append(_cache(), **kw) == code


def test_no_rows_at_all_need_no_gpu():
    assert _append(_cache(), cu=(0, 0, 0), k=None, v=None) == 0
    assert _read(_cache(), cu=(0, 0, 0), k=None, v=None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -5), (dict(B=65), -5), (dict(slots=(0, 4)), -1), (dict(slots=(2, 2)), -1), (dict(rows=None), -1), (dict(q=None), -1),
    (dict(out=None), -1), (dict(q=P + 8), -1), (dict(out=P + 2), -1), (dict(rows=P + 4), -1), (dict(mask=P + 4, mask_rows=3), -1),
    (dict(n_q=0), -5), (dict(n_q=65), -5), (dict(heads=3), -2), (dict(heads=0), -2), (dict(q_ld=252), -2), (dict(q_ld=248), -2),
    (dict(out_ld=257), -2), (dict(out_ld=128), -2), (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1),
    (dict(scale=float("inf")), -1), (dict(mask=P, mask_rows=0), -5), (dict(mask=P, mask_rows=1025), -5), (dict(dtype=7), -3),
])
def test_bad_inputs_of_attention_are_refused(kw, code):
    assert _attend(_cache(), **kw) == code


def test_the_reference_format_holds_every_value_within_half_a_step():
    import numpy as np
    from tests import kv4_reference as ref
    x = np.random.default_rng(0).standard_normal((50, 2, 64)).astype(np.float32)
    n, m, s = ref.quantise(x)
    assert np.all((n >= 0) & (n <= 15))
    step = np.repeat(s, 32, -1)
    assert np.all(np.abs(ref.values(n, m, s) - x) <= step / 2 * (1 + 1e-12))
    assert np.all(np.repeat(m, 32, -1) <= x) and np.all(np.repeat(m + 15 * s, 32, -1) >= x)
