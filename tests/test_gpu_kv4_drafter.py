"""Drafter contexts whose cache is held in 4 bits (dtype HIVIS_BF16_KV4): the rows that the prefix build and the draft steps leave,
the attention over them, the drafts, and a run of everything a server calls."""
import numpy as np
import pytest

import hivis_inputs as hi
from hivis_inputs.device import dev_weights, to_dev
from tests import kv4_reference as ref
from tests.harness import LOGIT_RTOL, row_rel_err

pytestmark = pytest.mark.gpu

NAMES = ["mini_mha_b5_ragged", "mini_gqa_b16_ragged", "gqa4_b5_ragged", "mini_mha_b1", "gqa2_b5_ragged"]


class Pair:
    """A workload in a context with a 4-bit cache and, where asked for, in one with a bf16 cache."""

    def __init__(self, wl, both=False, extra=None, max_k=None):
        import torch
        from paper_2509_23928_b200 import Drafter
        self.torch, self.wl, self.dims = torch, wl, wl.dims
        self.W = hi.make_weights(wl.dims, wl.seed)
        self.W.update(extra or {})
        self.ids, self.hidden, self.cu = hi.make_prompt(wl)
        self.resid = hi.make_residuals(wl)
        self.lens = np.diff(self.cu)
        dW = dev_weights(self.W, wl.dims.dtype)
        args = dict(max_batch=wl.batch, max_len=int(self.lens.max()) + 40, max_k=max_k or max(wl.k, 8))
        self.d4 = Drafter(wl.dims, dW, kv_bits=4, **args)
        self.d16 = Drafter(wl.dims, dW, **args) if both else None
        self.d_ids, self.d_hidden, self.d_resid = torch.from_numpy(self.ids).cuda(), to_dev(self.hidden, "bf16"), to_dev(self.resid, "bf16")

    def prefill(self, d):
        d.prefill(self.d_ids, self.d_hidden, [int(x) for x in self.cu], resid0=self.d_resid[0])

    def rows(self, d, b, n):
        k, v = d.read_kv(b, 0, n)
        self.torch.cuda.synchronize()
        shape = (n, self.dims.n_kv_heads, self.dims.head_dim)
        return k.cpu().numpy().reshape(shape).astype(np.float64), v.cpu().numpy().reshape(shape).astype(np.float64)

    def close(self):
        self.d4.close()
        if self.d16:
            self.d16.close()


def _rope(x, pos, base):
    """x [heads, dh] at a position."""
    half = x.shape[-1] // 2
    a = pos * base ** (-2.0 * np.arange(half) / x.shape[-1])
    lo, up = x[:, :half], x[:, half:]
    return np.concatenate([lo * np.cos(a) - up * np.sin(a), up * np.cos(a) + lo * np.sin(a)], -1)


def _steps(p, b, k, ids, K, V):
    """Logits [k, vocab] of sequence b's chain in 64 bits, its cached rows (those of the steps too) taken as K and V."""
    D, W = p.dims, {n: w.astype(np.float64) for n, w in p.W.items()}
    f, tok, pos = p.hidden[p.cu[b + 1] - 1].astype(np.float64), int(p.ids[p.cu[b + 1] - 1]), int(p.lens[b]) - 1
    group = D.n_q_heads // D.n_kv_heads
    out = []
    for s in range(k):
        u = W["fc"] @ np.concatenate([f, W["embed"][tok]]) + p.resid[min(s, len(p.resid) - 1)]
        a = u / np.sqrt((u * u).mean() + D.rms_eps) * W["norm1"]
        q = W["wq"] @ a + W.get("bq", 0.0)
        q = _rope(q.reshape(D.n_q_heads, D.head_dim), pos + s, D.rope_base)
        o = []
        for h in range(D.n_q_heads):
            z = K[:pos + s + 1, h // group] @ q[h] / np.sqrt(D.head_dim)
            w = np.exp(z - z.max())
            o.append(w @ V[:pos + s + 1, h // group] / w.sum())
        y = u + W["wo"] @ np.concatenate(o)
        m = y / np.sqrt((y * y).mean() + D.rms_eps) * W["norm2"]
        gate = W["w_gate"] @ m
        f = y + W["w_down"] @ (gate / (1.0 + np.exp(-gate)) * (W["w_up"] @ m))
        out.append(W["lm_head"] @ f)
        tok = int(ids[s])
    return np.stack(out)


def _biases(dims, seed):
    rng = np.random.default_rng(seed)
    return {n: hi.round_to_bf16((rng.standard_normal(w) * 0.5).astype(np.float32)) for n, w in
            (("bq", dims.q_dim), ("bk", dims.kv_dim), ("bv", dims.kv_dim))}


@pytest.mark.parametrize("gemms", [True, False])
@pytest.mark.parametrize("name", NAMES[:4])
def test_the_prefix_holds_what_a_bf16_cache_would_quantised(name, gemms):
    wl = hi.workload(name)
    p = Pair(wl, both=True, extra=_biases(wl.dims, 3))
    try:
        for d in (p.d4, p.d16):
            d.set_tc_prefill(2 if gemms else False)
            p.prefill(d)
        for b in range(wl.batch):
            n = int(p.lens[b]) - 1
            if n == 0:
                continue
            for got, x in zip(p.rows(p.d4, b, n), p.rows(p.d16, b, n)):
                codes, m, s = ref.quantise(x)
                want = ref.values(codes, m, s)
                # one fp32 operation on exact numbers
                assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want)), b
    finally:
        p.close()


@pytest.mark.parametrize("chain", ["tc", "phases"])
@pytest.mark.parametrize("name", NAMES)
def test_drafts_over_the_rows_that_are_held(name, chain):
    """The logits of every step against the step in 64 bits on the very rows that the cache holds."""
    wl = hi.workload(name)
    p = Pair(wl, extra=_biases(wl.dims, 4))
    try:
        p.d4.set_tc_kernel(chain == "tc")
        p.prefill(p.d4)
        ids, logits = p.d4.draft(wl.batch, wl.k, p.d_resid, want_logits=True)
        p.torch.cuda.synchronize()
        p.d4.status()
        ids, logits = ids.cpu().numpy(), logits.cpu().numpy()
        assert np.array_equal(ids, logits.argmax(-1))
        for b in range(wl.batch):
            n = int(p.lens[b]) - 1 + wl.k
            assert p.d4.kv_len(b) == (n, False)
            K, V = p.rows(p.d4, b, n)
            want = _steps(p, b, wl.k, ids[b], K, V)
            assert row_rel_err(logits[b], want).max() <= LOGIT_RTOL, b
        # the attention of the last step alone: queries as tapped (fp32), 11 bits of them and of the probabilities
        q, attn = (p.d4.tap(x, wl.batch).cpu().numpy().astype(np.float64) for x in ("q", "attn"))
        D = wl.dims
        for b in range(wl.batch):
            n = int(p.lens[b]) - 1 + wl.k
            K, V = p.rows(p.d4, b, n)
            rot = _rope(q[b].reshape(D.n_q_heads, D.head_dim), n - 1, D.rope_base)
            for h in range(D.n_q_heads):
                kk, vv = K[:, h // (D.n_q_heads // D.n_kv_heads)], V[:, h // (D.n_q_heads // D.n_kv_heads)]
                z = kk @ rot[h] / np.sqrt(D.head_dim)
                w = np.exp(z - z.max())
                w /= w.sum()
                terms = np.abs(kk) @ np.abs(rot[h]) / np.sqrt(D.head_dim)
                # a score is off by 2^-11 of its terms at most, a probability by as much and 2^-11 of itself
                reach = (w[:, None] * (np.abs(vv) + 15 * (np.abs(vv).max(0) / 7.5))).sum(0)
                tol = (2.0 ** -10 * (1.0 + terms.max())) * reach
                assert np.all(np.abs(attn[b].reshape(D.n_q_heads, D.head_dim)[h] - w @ vv) <= tol), (b, h)
    finally:
        p.close()


def test_the_two_ways_through_a_step_agree():
    wl = hi.workload("mini_mha_b5_ragged")
    p = Pair(wl)
    try:
        out = []
        for tc in (True, False):
            p.d4.set_tc_kernel(tc)
            p.prefill(p.d4) if not out else p.d4.set_kv_len_batch([int(x) - 1 for x in p.lens], restore_pending=True)
            forced = None if not out else out[0][0]
            ids, logits = p.d4.draft(wl.batch, wl.k, p.d_resid, forced_ids=forced, want_logits=True)
            out.append((ids, logits.cpu().numpy()))
        # (rows of the steps before may differ by a code where a value lies near a border: as far apart as two bf16 paths)
        assert row_rel_err(out[1][1], out[0][1]).max() <= 2 * LOGIT_RTOL
    finally:
        p.close()


@pytest.mark.parametrize("batch", [1, 2, 33, 64])
def test_any_batch(batch):
    wl = hi.scaled(hi.workload("mini_gqa_b3"), batch=batch, k=3, text_len=None, text_len_range=(1, 90))
    p = Pair(wl)
    try:
        p.prefill(p.d4)
        ids, logits = p.d4.draft(batch, 3, p.d_resid, want_logits=True)
        p.d4.status()
        ids, logits = ids.cpu().numpy(), logits.cpu().numpy()
        for b in sorted({0, batch // 2, batch - 1}):
            K, V = p.rows(p.d4, b, int(p.lens[b]) - 1 + 3)
            # (more than 16 sequences: activations are rounded to bf16 between the layers as well)
            assert row_rel_err(logits[b], _steps(p, b, 3, ids[b], K, V)).max() <= LOGIT_RTOL * (1 if batch <= 16 else 2), b
    finally:
        p.close()


@pytest.mark.parametrize("batch", [1, 5])
def test_drawn_and_forced_tokens(batch):
    wl = hi.scaled(hi.workload("mini_mha_b5_ragged"), batch=batch, k=4)
    p = Pair(wl)
    try:
        t, V = p.torch, wl.dims.vocab
        p.prefill(p.d4)
        u = t.empty((batch, 4, V), device="cuda").uniform_(1e-6, 1 - 1e-6)
        ids, logits = p.d4.draft_sampled(batch, 4, 0.8, u, p.d_resid)
        z = logits.double() / 0.8 - t.log(-t.log(u.double()))
        top = z.topk(2, -1)
        sure = top.values[..., 0] - top.values[..., 1] > 1e-4
        assert bool((ids.long() == top.indices[..., 0])[sure].all())
        p.d4.set_kv_len_batch([int(x) - 1 for x in p.lens], restore_pending=True)
        _, again = p.d4.draft(batch, 4, p.d_resid, forced_ids=ids, want_logits=True)
        assert t.equal(again, logits)
    finally:
        p.close()


def test_a_run_of_everything_a_server_calls():
    """Prefix, draft, how sure it is, verification, what is returned to the client, refresh of the accepted rows, draft again."""
    from paper_2509_23928_b200 import logprobs
    wl = hi.workload("gqa4_b5_ragged")
    p = Pair(wl)
    try:
        t, B, k, V = p.torch, wl.batch, wl.k, wl.dims.vocab
        p.prefill(p.d4)
        rows = [int(x) - 1 for x in p.lens]
        rng = np.random.default_rng(5)
        for turn in range(3):
            ids, logits = p.d4.draft(B, k, p.d_resid, want_logits=True)
            draft = logprobs(logits.view(B * k, V), ids.view(B * k, 1), top_n=3)
            # the chosen token is the most probable one, and its log-probability the largest
            assert t.equal(draft.top_ids[:, 0].view(B, k), ids) and t.equal(draft.logprobs[:, 0], draft.top_logprobs[:, 0])
            target, planted = hi.make_target_logits(hi.scaled(wl, seed=wl.seed + turn), ids.cpu().numpy())
            d_target = to_dev(target, wl.logits_dtype)
            acc, nxt, kv = p.d4.verify(ids, d_target)
            acc, nxt, kv = acc.tolist(), nxt, kv.tolist()
            assert acc == planted.tolist()
            assert kv == [r + 1 + min(n, k - 1) for r, n in zip(rows, acc)]
            # what the client gets: the committed tokens under the target's distributions
            committed = logprobs(d_target.view(B * (k + 1), V), t.cat([ids, nxt[:, None]], 1).view(-1, 1), top_n=1)
            top = committed.top_ids.view(B, k + 1)
            for b, n in enumerate(acc):
                assert top[b, :n].tolist() == ids[b, :n].tolist() and int(top[b, n]) == int(nxt[b])
            # the accepted rows are built again from the target's features, the next token becomes the pending one
            n_new = [n + 1 for n in acc]
            cu = [0] + [int(x) for x in np.cumsum(n_new)]
            tok = t.cat([t.cat([ids[b, :n], nxt[b:b + 1]]) for b, n in enumerate(acc)]).contiguous()
            hid = to_dev(hi.round_to_bf16(rng.standard_normal((cu[-1], wl.dims.d)).astype(np.float32)), "bf16")
            p.d4.prefill(tok, hid, cu, start_pos=[r + 1 for r in rows], resid0=p.d_resid[0])
            rows = [r + n + 1 for r, n in zip(rows, acc)]
            assert [p.d4.kv_len(b) for b in range(B)] == [(r, True) for r in rows]
        p.d4.status()
    finally:
        p.close()


def test_captured_turns_replay():
    wl = hi.workload("mini_mha_b5_ragged")
    p = Pair(wl)
    try:
        t, B, k = p.torch, wl.batch, wl.k
        p.prefill(p.d4)
        out = t.empty((B, k), dtype=t.int32, device="cuda")
        start = [int(x) - 1 for x in p.lens]

        def turn():
            p.d4.set_kv_len_batch(start, restore_pending=True)
            p.d4.draft(B, k, p.d_resid, out_ids=out)

        side = t.cuda.Stream()
        side.wait_stream(t.cuda.current_stream())
        with t.cuda.stream(side):
            turn()
        t.cuda.current_stream().wait_stream(side)
        want = out.clone()
        graph = t.cuda.CUDAGraph()
        with t.cuda.graph(graph):
            turn()
        for _ in range(3):
            out.zero_()
            graph.replay()
            assert t.equal(out, want)
        p.d4.status()
    finally:
        p.close()


def test_slots_in_any_order_and_rows_that_are_rebuilt():
    wl = hi.workload("mini_gqa_b3")
    p = Pair(wl)
    try:
        t = p.torch
        order = [2, 0, 1]
        p.d4.prefill(p.d_ids, p.d_hidden, [int(x) for x in p.cu], slots=order, resid0=p.d_resid[0])
        first = p.d4.draft(3, 2, p.d_resid, slots=order).clone()
        kept = [p.d4.read_kv(s, 0, 30) for s in range(3)]
        # back to 30 rows, the rest built again: the same drafts, the first rows untouched
        cut = [slice(int(c) + 30, int(c) + int(n)) for c, n in zip(p.cu[:-1], p.lens)]
        cu = [0] + [int(x) for x in np.cumsum([c.stop - c.start for c in cut])]
        p.d4.prefill(t.cat([p.d_ids[c] for c in cut]), t.cat([p.d_hidden[c] for c in cut]), cu, slots=order, start_pos=[30] * 3, resid0=p.d_resid[0])
        assert t.equal(p.d4.draft(3, 2, p.d_resid, slots=order), first)
        for s in range(3):
            assert all(t.equal(a, b) for a, b in zip(kept[s], p.d4.read_kv(s, 0, 30)))
    finally:
        p.close()


def test_what_such_a_context_does_not_do():
    from paper_2509_23928_b200 import Drafter, HivisError
    wl = hi.workload("mini_mha_b1")
    p = Pair(wl)
    try:
        p.prefill(p.d4)
        with pytest.raises(HivisError) as e:
            p.d4.draft_tree(0, 4, 3, 10, p.d_resid)
        assert e.value.code == -2
        p.d4.draft(1, 2, p.d_resid)                                  # nothing was launched, nothing has changed
        p.d4.status()
        rows, D = int(p.lens[0]), wl.dims
        assert p.d4.step_bytes([rows]) == D.step_params() * 2 + (rows + 1) * D.kv_dim * 5 // 4
        dW = dev_weights(p.W, "bf16")
        for bad in (8, 16, 2):
            with pytest.raises(ValueError):
                Drafter(wl.dims, dW, max_batch=1, max_len=32, kv_bits=bad)
        with pytest.raises(ValueError):
            Drafter(hi.workload("c1_tiny_f32_b1").dims, dW, max_batch=1, max_len=32, kv_bits=4)
    finally:
        p.close()


def test_a_missed_barrier_is_reported_and_survived():
    from paper_2509_23928_b200 import HivisError
    wl = hi.workload("mini_mha_b5_ragged")
    p = Pair(wl)
    try:
        p.prefill(p.d4)
        want = p.d4.draft(wl.batch, 2, p.d_resid).clone()
        p.d4.set_kv_len_batch([int(x) - 1 for x in p.lens], restore_pending=True)
        p.d4.set_wait_limit_us(2000)
        p.d4.miss_next_barrier()
        p.d4.draft(wl.batch, 2, p.d_resid)
        with pytest.raises(HivisError) as e:
            p.d4.status()
        assert e.value.code == -7
        p.d4.set_wait_limit_us(1000000)
        p.d4.set_kv_len_batch([int(x) - 1 for x in p.lens], restore_pending=True)
        assert p.torch.equal(p.d4.draft(wl.batch, 2, p.d_resid), want)
        p.d4.status()
    finally:
        p.close()
