"""What hivis_logprobs refuses before anything is launched (no GPU is touched)."""
import pytest

P = 0x10000


def _call(n=3, vocab=100, logits=P, dtype=0, ld=100, temperature=1.0, ids=P, n_ids=1, top=2, lp=P, h=P, top_ids=P, top_lp=P):
    from paper_2509_23928_b200.binding import lib
    return lib.hivis_logprobs(n, vocab, logits, dtype, ld, temperature, ids, n_ids, top, lp, h, top_ids, top_lp, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), -5), (dict(vocab=0), -2), (dict(vocab=2 ** 28 + 1, ld=2 ** 29), -2), (dict(dtype=2), -3), (dict(ld=99), -2),
    (dict(temperature=0.0), -1), (dict(temperature=-1.0), -1), (dict(temperature=float("nan")), -1), (dict(temperature=float("inf")), -1), (dict(temperature=1e-38), -1),
    (dict(n_ids=33), -5), (dict(n_ids=-1), -5), (dict(top=33), -5), (dict(top=-1), -5), (dict(logits=None), -1), (dict(ids=None), -1),
    (dict(lp=None), -1), (dict(top_ids=None), -1), (dict(top_lp=None), -1), (dict(logits=P + 4), -1), (dict(ids=P + 4), -1),
    (dict(h=P + 8), -1), (dict(top_lp=P + 2), -1), (dict(n_ids=0, top=0, h=None), -1),
])
def test_bad_arguments_are_refused(kw, code):
    from paper_2509_23928_b200 import hivis_last_error
    assert _call(**kw) == code
    assert "hivis_logprobs" in hivis_last_error(None)


def test_no_rows_need_no_gpu():
    assert _call(n=0, logits=None) == 0


@pytest.mark.parametrize("first", range(8))
def test_views_that_start_anywhere_are_copied_to_where_the_library_reads(first):
    import torch
    from paper_2509_23928_b200.binding import _aligned
    whole = torch.arange(8 * 40, dtype=torch.int32).view(8, 40)
    for t in (whole.view(-1)[first:first + 9], whole[:, first:first + 21], whole.bfloat16()[1:, first:], whole[:0, first:]):
        a = _aligned(t)
        assert a.data_ptr() % 16 == 0 and a.dtype is t.dtype and a.shape == t.shape and bool((a == t).all())
        assert a.numel() == 0 or a[0].is_contiguous()
        assert (a is t) == (t.data_ptr() % 16 == 0)
