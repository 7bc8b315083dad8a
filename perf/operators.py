"""The operators that a server has beside the drafter's own steps, as measurable cases.

  store     rows of keys and values go into a cache held in 4 bits, and are read back as the values it stands for: a
            prompt arrives, a step adds one position, a sequence is moved.
  attend    queries attend over such a cache: one position per sequence (a draft step), a block of k + 1 positions (the
            target's pass over a chain), the nodes of a draft tree under their ancestor mask.
  logprobs  log-probabilities of given tokens, the entropy and the top alternatives of rows of logits: what is returned to
            a client for the committed tokens, and what says how sure a draft is.

The 4-bit format, per row, KV head and group of 32 channels: m = the smallest value, rounded down to bf16; s = (the largest
- m) / 15, rounded up to bf16; every value is held as the nearest m + s n, n = 0..15, the lower one on a tie.
"""
import math

import torch

own = False

GROUP = 32


class Shape:
    """What the operators are told about a model."""

    def __init__(self, n_q_heads, n_kv_heads, head_dim, vocab):
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.vocab = n_q_heads, n_kv_heads, head_dim, vocab


SHAPES = {
    "tiny": Shape(4, 4, 64, 1024),            # the smallest drafter of the repository's configurations
    "llava": Shape(32, 32, 128, 32000),       # the two full-size ones: a KV head per query head,
    "qwen": Shape(28, 4, 128, 152064),        # and seven query heads to a KV head with a large vocabulary
    "mid": Shape(20, 4, 128, 50257),          # of no particular model: groups of five, rows of logits not aligned
    "gqa8": Shape(8, 1, 64, 3001),            # a reduced one: eight query heads on one KV head
}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"bf16": 2, "f32": 4}


def _store(name, shape, dtype, batch, lo, hi, start):
    """New rows per sequence of [lo, hi], behind up to `start` rows that are there already."""
    return {"name": name, "op": "store", "shape": shape, "dtype": dtype, "batch": batch, "lo": lo, "hi": hi, "start": start}


def _attend(name, shape, dtype, batch, lo, hi, n_q, tree=False):
    """Cached rows per sequence of [lo, hi], the n_q newest among them."""
    return {"name": name, "op": "attend", "shape": shape, "dtype": dtype, "batch": batch, "lo": lo, "hi": hi, "n_q": n_q, "tree": tree}


def _logprobs(name, shape, dtype, rows, n_ids, top, pad=0, banned=0.0, temperature=1.0):
    """`pad`: entries between the end of a row of logits and the next; `banned`: part of the vocabulary at -infinity."""
    return {"name": name, "op": "logprobs", "shape": shape, "dtype": dtype, "rows": rows, "n_ids": n_ids, "top": top, "pad": pad,
            "banned": banned, "temperature": temperature}


def listed():
    return [
        # one user: the position of one decoding step
        _store("store_llava_b1_token", "llava", "bf16", 1, 1, 1, 128),
        # a batch of prompts with uneven lengths, visual positions among them
        _store("store_llava_b16_prompts", "llava", "bf16", 16, 64, 704, 0),
        # the smallest attention: one short sequence, fp32
        _attend("attend_tiny_f32_b1", "tiny", "f32", 1, 32, 32, 1),
        # a draft step of a small server's batch, every sequence of its own length
        _attend("attend_llava_b16_ragged", "llava", "bf16", 16, 64, 512, 1),
        # a draft step of a batch with 2048 visual positions per sequence
        _attend("attend_llava_b16_visual", "llava", "bf16", 16, 2176, 2176, 1),
        # a few long documents, grouped heads
        _attend("attend_qwen_b4_long", "qwen", "bf16", 4, 9001, 32768, 1),
        # the target's pass over a chain of seven drafted tokens
        _attend("attend_qwen_b8_block", "qwen", "bf16", 8, 1024, 4096, 8),
        # the target's pass over a draft tree of 60 nodes and its root, 2048 visual positions before it
        _attend("attend_llava_tree", "llava", "bf16", 1, 2237, 2237, 61, tree=True),
        # one user: the rows of a verified chain of five, five alternatives for each
        _logprobs("logprobs_llava_b1", "llava", "bf16", 6, 1, 5),
        # the drafter's own rows of a batch, fp32, no alternatives: is the draft worth verifying?
        _logprobs("logprobs_qwen_b8_entropy", "qwen", "f32", 56, 1, 0),
        # a prompt is scored: many rows, not aligned, some tokens banned
        _logprobs("logprobs_mid_prompt", "mid", "f32", 1021, 1, 1, banned=0.3),
        # the largest: a full batch's verified chains with twenty alternatives, at a temperature
        _logprobs("logprobs_qwen_b64_top20", "qwen", "bf16", 64 * 8, 2, 20, pad=64, temperature=0.7),
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "attend", "attend", "attend", "logprobs", "logprobs"])
    shape = rng.choice(["llava", "qwen", "mid", "tiny", "gqa8"])
    S = SHAPES[shape]
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    values = S.n_kv_heads * S.head_dim                       # of a row of keys
    if op == "store":
        batch = _spread(rng, 1, 64)
        hi = _spread(rng, 1, max(1, min(4096, 20_000_000 // (values * batch))))
        return _store(None, shape, dtype, batch, rng.randint(1, hi), hi, rng.choice([0, rng.randint(1, 300)]))
    if op == "attend":
        batch = _spread(rng, 1, 64)
        tree = rng.random() < 0.2
        n_q = 1 if rng.random() < 0.5 else rng.randint(2, 61 if tree else 17)
        hi = _spread(rng, 1, min(32768, 140_000_000 // (values * batch), 300_000_000 // (batch * S.n_q_heads * n_q)))
        return _attend(None, shape, dtype, batch, rng.randint(1 + hi // 8, hi) if rng.random() < 0.7 else hi, hi, n_q, tree)
    rows = _spread(rng, 1, min(4096, 70_000_000 // S.vocab))
    return _logprobs(None, shape, dtype, rows, rng.choice([1, 1, 2, 5]), rng.choice([0, 1, 5, 20]), rng.choice([0, 0, 1, 64]),
                     rng.choice([0.0, 0.0, 0.3]), rng.choice([1.0, 1.0, 0.7, 1.5]))


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(case, gen):
    """Spread evenly over [lo, hi]; which sequence has which is drawn."""
    lo, span, n = case["lo"], case["hi"] - case["lo"], case["batch"]
    even = [lo + int(span * (b + 0.5) / n) for b in range(n)]
    return [even[b] for b in torch.randperm(n, generator=gen).tolist()]


def _kv(S, rows, dtype, gen):
    """Keys (a few channels of a head far off centre, as a model's are) and values of `rows` positions."""
    shape = (rows, S.n_kv_heads, S.head_dim)
    offset = torch.empty((1,) + shape[1:], device="cuda").normal_(0.0, 1.0, generator=gen)
    k = torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=gen).add_(offset * offset.abs())
    v = torch.empty(shape, device="cuda").normal_(0.0, 1.0, generator=gen)
    return k.to(TYPES[dtype]), v.to(TYPES[dtype])


def _starts(counts):
    cu = [0]
    for n in counts:
        cu.append(cu[-1] + n)
    return cu


def _tree_mask(batch, n, gen):
    """Who sees whom among the n newest rows: row 0 is the root, every later one hangs on an earlier one; true: visible."""
    up = torch.zeros((batch, n, n), dtype=torch.bool)
    for b in range(batch):
        for i in range(n):
            if i:
                up[b, i] = up[b, int(torch.randint(0, i, (1,), generator=gen))]
            up[b, i, i] = True
    return up


def _words(mask):
    """[B, n_q, T] truth values as 32-bit words, bit j of word w for row 32 w + j."""
    B, n_q, T = mask.shape
    w = (T + 31) // 32
    padded = torch.zeros((B, n_q, w * 32), dtype=torch.int64)
    padded[..., :T] = mask
    words = (padded.view(B, n_q, w, 32) << torch.arange(32)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def _inputs(case, seed):
    """Everything an operator is given, from the seed alone."""
    S, op = SHAPES[case["shape"]], case["op"]
    host = torch.Generator().manual_seed(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = TYPES[case["dtype"]]
    if op == "logprobs":
        n, V = case["rows"], S.vocab
        # rows of every temper: from nearly flat to nearly certain
        x = torch.empty((n, V + case["pad"]), device="cuda").normal_(0.0, 1.0, generator=gen)
        x *= torch.empty((n, 1), device="cuda").uniform_(0.5, 5.0, generator=gen)
        if case["banned"]:
            x.masked_fill_(torch.empty((1, V + case["pad"]), device="cuda").uniform_(0.0, 1.0, generator=gen) < case["banned"], -math.inf)
        # the tokens asked for: one of the likelier ones and others
        x = x.to(dtype)[:, :V]
        ids = torch.randint(0, V, (n, case["n_ids"]), generator=gen, device="cuda", dtype=torch.int32)
        ids[:, 0] = x[:, : max(1, V // 50)].argmax(-1).int()
        return {"logits": x, "ids": ids}
    T = _lengths(case, host)
    k, v = _kv(S, sum(T), case["dtype"], gen)
    if op == "store":
        start = torch.randint(0, case["start"] + 1, (case["batch"],), generator=host).tolist()
        return {"T": T, "k": k, "v": v, "start": start}
    q = torch.empty((case["batch"] * case["n_q"], S.n_q_heads, S.head_dim), device="cuda").normal_(0.0, 1.5, generator=gen).to(dtype)
    mask = _tree_mask(case["batch"], case["n_q"], host) if case["tree"] else None
    return {"T": T, "k": k, "v": v, "q": q, "mask": mask}


# -------------------------------------------------------------------------------------------------------- plain forms
def _quantise(x):
    """[..., dh] -> (codes 0..15 as bytes, m, s as bf16 per group of 32 channels).  In 64 bits: which code is nearest, and
    which bf16 value lies next above, are decided there without error."""
    g = x.double().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    m = lo.to(torch.bfloat16)
    m = torch.where(m.double() > lo, torch.nextafter(m, torch.full_like(m, -math.inf)), m)
    step = (hi - m.double()) / 15.0
    s = step.to(torch.bfloat16)
    s = torch.where(s.double() < step, torch.nextafter(s, torch.full_like(s, math.inf)), s)
    t = (g - m.double()[..., None]) / s.double()[..., None]
    n = torch.ceil(t - 0.5).clamp(0.0, 15.0).nan_to_num(0.0)       # (0 / 0: a group of equal values)
    return n.flatten(-2).to(torch.uint8), m, s


def _pack(n):
    return n[..., 0::2] | (n[..., 1::2] << 4)


def _values(packed, m, s):
    """The fp32 values that packed codes stand for."""
    n = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).float()
    return (n.unflatten(-1, (-1, GROUP)) * s.float()[..., None] + m.float()[..., None]).flatten(-2)


def _plain_cache(n_slots, n_kv_heads, head_dim, max_len):
    def zeros(last, dtype):
        return torch.zeros((n_slots, max_len, n_kv_heads, last), dtype=dtype, device="cuda")
    return [[zeros(head_dim // 2, torch.uint8), zeros(head_dim // GROUP, torch.bfloat16), zeros(head_dim // GROUP, torch.bfloat16)]
            for _ in range(2)]


def _plain_store(cache, slot, row, k, v):
    for held, x in zip(cache, (k, v)):
        n, m, s = _quantise(x)
        held[0][slot, row], held[1][slot, row], held[2][slot, row] = _pack(n), m, s


def _plain_read(cache, slot, row):
    return [_values(*(a[slot, row] for a in held)) for held in cache]


def _plain_attend(state):
    k, v = (_values(*held) for held in state["cache"])               # [B, L, Hkv, dh]
    q, rows, n_q = state["q"], state["rows"].long(), state["n_q"]
    B, L, Hkv, dh = k.shape
    Hq = q.shape[1]
    r = torch.arange(L, device="cuda")
    at = rows[:, None] - n_q                                          # first of the newest rows
    if state["mask"] is None:
        seen = r[None, None] <= (at + torch.arange(n_q, device="cuda"))[..., None]
    else:
        j = r[None] - at                                              # [B, L]: which of the newest rows
        word = state["mask"].long()[..., ((torch.arange(n_q, device="cuda")) // 32)]
        bit = (word >> (torch.arange(n_q, device="cuda") % 32)) & 1   # [B, n_q, n_q]
        newest = torch.gather(bit, 2, j.clamp(0, n_q - 1)[:, None].expand(B, n_q, L)) > 0
        seen = torch.where((j < 0)[:, None], True, newest & (r[None] < rows[:, None])[:, None])
    x = q.float().view(B, n_q, Hkv, Hq // Hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, dh)
    z = torch.matmul(x, k.permute(0, 2, 3, 1)).div_(math.sqrt(dh)).view(B, Hkv, -1, n_q, L)
    z = z.masked_fill_(~seen[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z.sub_(top.masked_fill_(top == -math.inf, 0.0)))
    total = e.sum(-1, keepdim=True)
    p = e / total.masked_fill_(total == 0.0, 1.0)                      # nothing to see: zeros
    o = torch.matmul(p.view(B, Hkv, -1, L), v.permute(0, 2, 1, 3)).view(B, Hkv, -1, n_q, dh)
    return o.permute(0, 3, 1, 2, 4).reshape(B * n_q, Hq, dh).to(q.dtype)


def _plain_logprobs(logits, ids, temperature, top_n):
    x = logits.float()
    top = x.amax(-1, keepdim=True)
    y = (x - torch.where(top == -math.inf, 0.0, top)) / temperature
    e = torch.exp(y)
    z = e.sum(-1, keepdim=True)
    log_z = torch.log(z)
    out = {"logprobs": torch.where(z > 0.0, y.gather(1, ids.long()) - log_z, -math.inf)}
    weighted = torch.where(e > 0.0, e * y, 0.0).sum(-1)
    out["entropy"] = torch.where(z[:, 0] > 0.0, log_z[:, 0] - weighted / z[:, 0], 0.0)
    if top_n:
        # by value, the lowest token among equals: one whole number that is in that order; -1 where no token is left
        bits = (x + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -2 ** 31 - 1 - bits)     # (the bits of a negative number fall as it rises)
        key = order * 2 ** 20 + (2 ** 20 - 1 - torch.arange(x.shape[1], device="cuda"))
        best = 2 ** 20 - 1 - (key.topk(top_n, dim=-1).values & (2 ** 20 - 1))
        mass = x.gather(1, best) > -math.inf
        out["top_ids"] = torch.where(mass, best, -1).int()
        out["top_logprobs"] = torch.where(mass, y.gather(1, best) - log_z, -math.inf)
    return out


# -------------------------------------------------------------------------------------------------------------- state
def prepare(case, seed):
    S, op = SHAPES[case["shape"]], case["op"]
    x = _inputs(case, seed)
    if op == "logprobs":
        return {"op": op, "logits": x["logits"], "ids": x["ids"], "temperature": case["temperature"], "top": case["top"]}
    B, T = case["batch"], x["T"]
    start = x.get("start") or [0] * B
    longest = (max(a + n for a, n in zip(start, T)) + 31) // 32 * 32
    cu = _starts(T)
    first = torch.tensor(start, dtype=torch.int32, device="cuda")
    if own:
        from paper_2509_23928_b200 import Kv4Cache
        cache = Kv4Cache(B, S.n_kv_heads, S.head_dim, longest)
    else:
        cache = _plain_cache(B, S.n_kv_heads, S.head_dim, longest)
        slot = torch.repeat_interleave(torch.arange(B), torch.tensor(T)).cuda()
        row = torch.cat([torch.arange(a, a + n) for a, n in zip(start, T)]).cuda()
    st = {"op": op, "cache": cache, "cu": cu, "first": first}
    if op == "store":
        st.update(k=x["k"], v=x["v"])
        if not own:
            st.update(slot=slot, row=row)
        return st
    if own:
        cache.append(x["k"], x["v"], cu, first)
    else:
        for b in range(B):                                            # one sequence at a time: 64 bits take room
            i = slice(cu[b], cu[b + 1])
            _plain_store(cache, slot[i], row[i], x["k"][i], x["v"][i])
    st.update(q=x["q"], rows=torch.tensor(T, dtype=torch.int32, device="cuda"), n_q=case["n_q"],
              mask=None if x["mask"] is None else _words(x["mask"]).cuda())
    return st


def run(state):
    op = state["op"]
    if op == "logprobs":
        if own:
            from paper_2509_23928_b200 import logprobs
            out = logprobs(state["logits"], state["ids"], temperature=state["temperature"], top_n=state["top"])
            return {name: t for name, t in out._asdict().items() if t is not None}
        return _plain_logprobs(state["logits"], state["ids"], state["temperature"], state["top"])
    cache = state["cache"]
    if op == "store":
        if own:
            cache.append(state["k"], state["v"], state["cu"], state["first"])
            k, v = cache.read(state["cu"], state["first"])
        else:
            _plain_store(cache, state["slot"], state["row"], state["k"], state["v"])
            k, v = _plain_read(cache, state["slot"], state["row"])
        return {"k": k, "v": v}
    if own:
        if state["mask"] is None:
            return cache.attention(state["q"], state["rows"], n_q=state["n_q"])
        return cache.attention(state["q"], state["rows"], n_q=state["n_q"], mask=state["mask"], mask_rows=state["n_q"])
    return _plain_attend(state)


def work(case):
    """store: the rows read, the cache written and read, the values written.  attend: every cached row and the queries read
    once, the results written; both products for every visible pair.  logprobs: every logit read once."""
    S, op = SHAPES[case["shape"]], case["op"]
    size = SIZES[case["dtype"]]
    if op == "logprobs":
        n = case["rows"]
        return {"bytes": n * (S.vocab * size + 4.0 * (2 * case["n_ids"] + 1 + 2 * case["top"])), "flops": 5.0 * n * S.vocab}
    mean = (case["lo"] + case["hi"]) / 2
    values = 2.0 * case["batch"] * mean * S.n_kv_heads * S.head_dim    # of keys and values
    held = 0.5 + 4.0 / GROUP                                          # bytes a value
    if op == "store":
        return {"bytes": values * (size + 2 * held + 4), "flops": 8.0 * values}
    nodes = case["batch"] * case["n_q"]
    return {"bytes": values * held + 2.0 * nodes * S.n_q_heads * S.head_dim * size,
            "flops": 4.0 * nodes * S.n_q_heads * S.head_dim * max(1.0, mean - case["n_q"] / 2)}


# -------------------------------------------------------------------------------------------------------------- exact
def _held_exactly(x):
    """The values that the 4-bit format holds for x [..., dh], in 64 bits: a grid of 16 points per group of 32 channels."""
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], GROUP):
        part = x[..., c:c + GROUP]
        low, high = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
        base = _to_bf16(low, torch.floor)
        step = _to_bf16((high - base) / 15, torch.ceil)
        # steps from the base, a half counted down; groups of equal values have no step
        steps = torch.where(step > 0, -torch.floor(0.5 - (part - base) / torch.where(step > 0, step, 1.0)), 0.0)
        out[..., c:c + GROUP] = base + step * steps.clamp(0, 15)
    return out


def _to_bf16(x, rounding):
    """x to 8 significant bits (numbers far from the ends of bf16's range), in the direction of `rounding`."""
    frac, exp = torch.frexp(x)
    return torch.ldexp(rounding(frac * 256.0), exp - 8)


@torch.no_grad()
def exact(case, seed):
    S, op = SHAPES[case["shape"]], case["op"]
    x = _inputs(case, seed)
    if op == "logprobs":
        n = case["rows"]
        lp = torch.empty((n, case["n_ids"]), dtype=torch.float64, device="cuda")
        ent = torch.empty((n,), dtype=torch.float64, device="cuda")
        tlp = torch.empty((n, case["top"]), dtype=torch.float64, device="cuda")
        for a in range(0, n, 64):
            # (the temperature is a 32-bit number for the operator, but exact to 1e-7 of itself, which a logarithm keeps)
            all_lp = torch.log_softmax(x["logits"][a:a + 64].double() / case["temperature"], -1)
            lp[a:a + 64] = all_lp.gather(1, x["ids"][a:a + 64].long())
            ent[a:a + 64] = torch.special.entr(all_lp.exp()).sum(-1)
            if case["top"]:
                tlp[a:a + 64] = all_lp.sort(-1, descending=True).values[:, :case["top"]]
        out = {"logprobs": lp, "entropy": ent}
        if case["top"]:
            out.update(top_ids=None, top_logprobs=tlp)
        return out
    if op == "store":
        return {"k": _held_exactly(x["k"]), "v": _held_exactly(x["v"])}
    B, n_q, T = case["batch"], case["n_q"], x["T"]
    cu = _starts(T)
    q = x["q"].double().view(B, n_q, S.n_kv_heads, -1, S.head_dim)
    out = torch.zeros_like(q)
    for b in range(B):
        for h in range(S.n_kv_heads):
            k, v = (_held_exactly(x[m][cu[b]:cu[b + 1], h]) for m in "kv")
            see = torch.ones((n_q, T[b]), dtype=torch.bool, device="cuda").tril(T[b] - n_q)
            if x["mask"] is not None:
                new = min(n_q, T[b])                                  # a short sequence holds the last rows of its tree only
                see = torch.ones_like(see)
                see[:, T[b] - new:] = x["mask"][b, :, n_q - new:].cuda()
            z = torch.einsum("igd,rd->igr", q[b, :, h], k) / math.sqrt(S.head_dim)
            w = torch.softmax(z.masked_fill(~see[:, None], -math.inf), -1).nan_to_num(0.0)
            out[b, :, h] = torch.einsum("igr,rd->igd", w, v)
    return out.reshape(B * n_q, S.n_q_heads, S.head_dim)
