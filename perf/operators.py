"""Work on caches whose instances have lengths of their own: appending rows, attention of one new token, attention of a
chunk of new tokens, and eviction by accumulated attention weight, call by call.

A case is one call at one size.  An instance is one (layer, batch, KV head) triple; the instances of a sequence share its
length.  Pages are those of a pool in which they lie in any order, or the cache is contiguous.  The kinds ("op"):

  append   the K/V rows of the new tokens go to their places in the cache (Context.cache_append)
  decode   one new token per sequence over its whole cache, or over a window and the first tokens (Context.cache_decode)
  prefill  a chunk of new tokens per sequence, each of which sees what lies before it (Context.cache_prefill)
  evict    caches beyond their budget keep their first rows, their last rows and the heaviest between (Context.cache_evict)

With `weights`, decode and prefill also add every row's attention weight, over the heads and queries, to what it gathered so far.

run() has each of them in its plain form, in 32 bits, and, where `own` is set, as the library's call.
"""
import math

import torch

own = False

_BASE = {"op": "decode", "seqs": 1, "heads": 8, "g": 4, "d": 128, "block": 16, "dtype": "bf16", "paged": True, "lo": 2000, "hi": 2048,
         "q": 1, "window": 0, "first": 0, "weights": False, "budget": 0, "last": 0}


def _case(name, **kw):
    return dict(_BASE, name=name, **kw)


def listed():
    return [
        # One layer of an 8B-shaped model, one sequence: the row of a decode step. Nothing but launch and latency.
        _case("append_one_row", op="append", lo=2040, hi=2040),
        # Prefill chunks of 16 sequences of such a layer, of different lengths.
        _case("append_chunks", op="append", seqs=16, lo=2100, hi=30000, q=2048),
        # One layer, one sequence of moderate length: the latency of a decode step that reads its whole cache.
        _case("decode_one_seq", lo=2041, hi=2041),
        # A batch of 32 sequences of very different lengths in one layer.
        _case("decode_ragged_batch", seqs=32, lo=60, hi=32790),
        # 70B-like grouping, two layers in a call, a sliding window with a few first tokens kept: what lies between is not read.
        _case("decode_window", seqs=128, heads=8, g=8, block=32, lo=3000, hi=16400, window=4096, first=4),
        # A cache under a budget, which gathers the weights that the eviction goes by.
        _case("decode_weights", seqs=32, lo=1025, hi=8190, weights=True),
        # The tiny fp32 shape of the tests, contiguous, weights gathered.
        _case("decode_tiny_f32", seqs=1, heads=1, d=64, dtype="f32", paged=False, lo=2049, hi=2049, weights=True),
        # A short prompt's tail behind a cached prefix.
        _case("prefill_short", op="prefill", lo=517, hi=517, q=101),
        # A whole prompt of one layer, every query sees all before it.
        _case("prefill_prompt", op="prefill", lo=8190, hi=8190, q=8190),
        # Chunks of two sequences behind long caches, sliding window and first tokens.
        _case("prefill_window", op="prefill", seqs=2, block=32, lo=9001, hi=16390, q=2048, window=2048, first=4, weights=True),
        # After a prompt: caches of 2 to 32 thousand rows go down to a budget of 1024.
        _case("evict_prompt", op="evict", seqs=8, lo=2050, hi=32790, budget=1024, first=64, last=64),
        # While decoding, four layers in a call: every 64 steps the rows beyond the budget leave.
        _case("evict_steady", op="evict", seqs=32, lo=1088, hi=1088, budget=1024, first=64, last=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_BASE, op=rng.choice(["append", "decode", "decode", "decode", "prefill", "prefill", "prefill", "evict", "evict"]))
    c["heads"] = rng.choice([1, 2, 8, 8, 8, 32])
    c["g"] = rng.choice([1, 2, 4, 4, 4, 8])
    c["d"] = rng.choice([64, 128, 128])
    c["block"] = rng.choice([8, 16, 16, 32, 64])
    c["dtype"] = rng.choice(["f32", "bf16", "bf16", "bf16", "bf16"])
    c["paged"] = rng.random() < 0.7
    c["hi"] = _log_int(rng, 40, 32000)
    c["lo"] = max(1, int(c["hi"] * rng.choice([0.02, 0.3, 0.9, 1.0])))
    size = 2 if c["dtype"] == "bf16" else 4
    most = {"append": 3.0e9, "evict": 0.5e9}.get(c["op"], 1.0e9) / (c["hi"] * c["d"] * size)      # instances: bounded by the bytes of K ...
    if c["op"] in ("append", "prefill"):
        c["q"] = min(c["hi"], _log_int(rng, 1, 8192))
    if c["op"] == "append":
        most = min(most, 0.5e9 / (c["q"] * c["d"] * size))
    if c["op"] == "prefill":                                  # ... and by the scores of the plain form
        c["q"] = max(1, min(c["q"], int(4e8 / (c["g"] * c["hi"]))))
        most = min(most, 1.0e9 / (c["q"] * c["g"] * c["hi"]))
    if c["op"] in ("decode", "prefill"):
        c["window"] = rng.choice([0, 0, max(1, int(c["hi"] * rng.uniform(0.05, 0.9)))])
        c["first"] = rng.choice([0, 1, 4, 37]) if c["window"] else 0
        c["weights"] = rng.random() < 0.5
    if c["op"] == "evict":
        c["budget"] = max(8, int(c["hi"] * rng.uniform(0.03, 0.95)))
        c["first"] = rng.choice([0, 4, c["budget"] // 16])
        c["last"] = rng.choice([1, c["budget"] // 4, c["budget"] // 2])
    c["seqs"] = max(1, min(256, _log_int(rng, 1, max(1.0, most / c["heads"]))))
    return c


# ------------------------------------------------------------------------------------------------------------------
# Sizes, from the case alone; the seed only says which sequence has which length
# ------------------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n whole numbers from lo to hi, even over their logarithm, hi among them."""
    if n == 1:
        return [hi]
    at = [((k * 0.6180339887498949) % 1.0) for k in range(n - 1)]
    return [hi] + [max(1, min(hi, int(round(lo * (hi / lo) ** u)))) for u in at]


def _lengths(c):
    """Length of each sequence's cache, and its new tokens."""
    lens = _spread(c["seqs"], c["lo"], c["hi"])
    new = _spread(c["seqs"], max(1, (2 * c["q"]) // 3), c["q"])
    return lens, [min(a, b) for a, b in zip(new, lens)]


def _cap(c):
    return -(-(c["hi"] + 1) // 64) * 64


def _seen(c, p):
    """Rows that a query at position p sees."""
    if not c["window"]:
        return p + 1
    return min(p + 1, c["window"]) + max(0, min(c["first"], p + 1 - c["window"]))


def work(case):
    c = case
    lens, new = _lengths(c)
    row = c["d"] * (2 if c["dtype"] == "bf16" else 4)
    h, g = c["heads"], c["g"]
    tables = (lambda rows: 4 * rows / c["block"]) if c["paged"] else (lambda rows: 0)
    if c["op"] == "append":
        return {"bytes": h * (4 * row * sum(new) + tables(sum(new)) + 8 * len(lens)), "flops": 0}
    if c["op"] == "decode":
        rows = sum(_seen(c, n - 1) for n in lens)
        return {"bytes": h * (rows * (2 * row + (8 if c["weights"] else 0)) + tables(rows) + len(lens) * (g * (row + 4 * c["d"]) + 4)),
                "flops": 4 * h * g * c["d"] * rows}
    if c["op"] == "prefill":
        pairs = sum(_seen(c, n - k + r) for n, k in zip(lens, new) for r in range(k))
        rows = sum(n if not c["window"] else min(n, c["window"] + k - 1 + c["first"]) for n, k in zip(lens, new))
        return {"bytes": h * (rows * (2 * row + (8 if c["weights"] else 0)) + tables(rows) + 2 * g * row * sum(new) + 8 * len(lens)),
                "flops": 4 * h * g * c["d"] * pairs}
    over = [n for n in lens if n > c["budget"]]
    return {"bytes": h * (4 * row * c["budget"] * len(over) + 4 * sum(over) + 4 * sum(over) + 4 * sum(min(n, c["budget"]) for n in lens) + 8 * len(lens)),
            "flops": 0}


# ------------------------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------------------------
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _normal(shape, c, seed, what, scale=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed((int(seed) * 1000003 + what * 7919 + 12345) % (1 << 62))
    x = torch.empty(shape, dtype=_dtype(c), device="cuda").normal_(generator=gen)
    return x if scale == 1.0 else x.mul_(scale)


def prepare(case, seed):
    c = case
    n, cap, b, d = c["seqs"] * c["heads"], _cap(c), c["block"], c["d"]
    lens, new = _lengths(c)
    turn = int(seed) % len(lens)
    lens, new = lens[turn:] + lens[:turn], new[turn:] + new[:turn]
    per = lambda v: torch.tensor([x for x in v for _ in range(c["heads"])], dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"c": c, "cap": cap, "len": per(lens), "new": per(new), "table": None}
    gen = torch.Generator(device="cuda")
    gen.manual_seed((int(seed) * 1000003 + 777) % (1 << 62))
    if c["paged"]:
        s["table"] = torch.randperm(n * (cap // b), generator=gen, device="cuda").to(torch.int32).view(n, cap // b)
    shape = (n * (cap // b), b, d) if c["paged"] else (n, cap, d)
    s["K"], s["V"] = _normal(shape, c, seed, 1), _normal(shape, c, seed, 2)
    if c["op"] == "append":
        s["k_new"], s["v_new"] = _normal((n, c["q"], d), c, seed, 3), _normal((n, c["q"], d), c, seed, 4)
    if c["op"] in ("decode", "prefill"):
        # Queries of twice the keys' size: scores spread by two, so that few rows carry most of the weight.
        lead = (n, c["g"], d) if c["op"] == "decode" else (n, c["q"], c["g"], d)
        s["q"] = _normal(lead, c, seed, 5, 2.0)
        s["out"] = torch.zeros(lead, dtype=torch.float32 if c["op"] == "decode" else _dtype(c), device="cuda")
    s["acc"] = None
    if c["weights"] or c["op"] == "evict":
        # What rows gathered so far: a few have most of it, and the newest have nothing yet.
        s["acc"] = torch.empty((n, cap), device="cuda").normal_(generator=gen).mul_(2.0).exp_()
        at = torch.arange(cap, device="cuda")[None, :]
        s["acc"] *= at < (s["len"] - torch.where(s["len"] > 40, 16, 0))[:, None]
    if c["op"] == "evict":
        s["acc_out"], s["len_out"] = torch.zeros_like(s["acc"]), torch.zeros_like(s["len"])
        s["kept"] = torch.full((n, c["budget"]), -1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2502_04077_amd import Context
        s["ctx"] = Context(n_inst=n, g=c["g"], head_dim=d, block=b, hist_len=1, t_cap=cap, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4,
                           kv_dtype=c["dtype"])
        if c["paged"]:
            s["ctx"].set_block_table(s["table"], n * (cap // b))
        size = s["ctx"].cache_workspace_bytes(c["q"] if c["op"] == "prefill" else 0, c["weights"])
        s["ws"] = torch.zeros(max(16, size), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------------------------
def _place(s, at):
    """Rows of the pool, seen as [rows][d], at which rows `at` [n][m] of the caches lie."""
    c, n = s["c"], s["len"].shape[0]
    at = at.long()
    if s["table"] is None:
        return torch.arange(n, device="cuda")[:, None] * s["cap"] + at
    return s["table"].long().gather(1, at // c["block"]) * c["block"] + at % c["block"]


def _rows(s, which, n_rows):
    """The first n_rows rows of every cache, in 32 bits: [n][n_rows][d]."""
    c, n = s["c"], s["len"].shape[0]
    at = torch.arange(n_rows, device="cuda")[None, :].expand(n, n_rows)
    return s[which].view(-1, c["d"])[_place(s, at)].float()


def _visible(s, pos, n_rows):
    """pos [n][m]: positions of queries; which rows each sees, [n][m][n_rows]."""
    c = s["c"]
    j = torch.arange(n_rows, device="cuda")[None, None, :]
    p = pos[:, :, None]
    seen = j <= p
    if c["window"]:
        seen = seen & ((j > p - c["window"]) | (j < c["first"]))
    return seen


def _attend(s, q, pos, n_rows):
    """q [n][m][g][d] at positions pos [n][m]: outputs [n][m][g][d] and probabilities [n][m][g][n_rows]."""
    n, m, g, d = q.shape
    K, V = _rows(s, "K", n_rows), _rows(s, "V", n_rows)
    w = torch.matmul(q.float().view(n, m * g, d), K.transpose(1, 2).contiguous()).view(n, m, g, n_rows)
    w = w.mul_(1.0 / math.sqrt(d)).masked_fill_(~_visible(s, pos, n_rows)[:, :, None, :], -math.inf)
    top = w.amax(-1, keepdim=True)
    w = w.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = w.sum(-1, keepdim=True)
    w = w.div_(torch.where(total == 0, 1.0, total))
    return torch.matmul(w.view(n, m * g, n_rows), V).view(n, m, g, d), w


def _plain_append(s):
    c = s["c"]
    r = torch.arange(c["q"], device="cuda")[None, :]
    at = (s["len"] - s["new"])[:, None] + r
    good = r < s["new"][:, None]
    to = _place(s, at.clamp(0, s["cap"] - 1))[good]
    s["K"].view(-1, c["d"])[to] = s["k_new"][good]
    s["V"].view(-1, c["d"])[to] = s["v_new"][good]
    return [s["K"], s["V"]]


def _plain_decode(s):
    out, w = _attend(s, s["q"][:, None], s["len"][:, None] - 1, s["c"]["hi"])
    s["out"].copy_(out[:, 0])
    if s["c"]["weights"]:
        s["acc"][:, :s["c"]["hi"]] += w.sum((1, 2))
        return [s["out"], s["acc"]]
    return [s["out"]]


def _plain_prefill(s):
    c = s["c"]
    r = torch.arange(c["q"], device="cuda")[None, :]
    good = r < s["new"][:, None]
    out, w = _attend(s, s["q"], (s["len"] - s["new"])[:, None] + r, c["hi"])
    s["out"].copy_(torch.where(good[:, :, None, None], out.to(s["out"].dtype), s["out"]))
    if c["weights"]:
        s["acc"][:, :c["hi"]] += (w.sum(2) * good[:, :, None]).sum(1)
        return [s["out"], s["acc"]]
    return [s["out"]]


def _plain_evict(s):
    c, cap, L = s["c"], s["cap"], s["len"].long()[:, None]
    j = torch.arange(cap, device="cuda")[None, :]
    forced = (j < c["first"]) | (j >= L - c["last"])
    rank = torch.where(forced, math.inf, s["acc"]).masked_fill(j >= L, -math.inf)
    best = rank.sort(dim=1, descending=True, stable=True)[1][:, :c["budget"]].sort(dim=1)[0]
    slot = torch.arange(c["budget"], device="cuda")[None, :]
    best = torch.where(L > c["budget"], best, slot.expand_as(best))
    left = torch.minimum(L, torch.tensor(c["budget"], device="cuda"))
    real = slot < left
    src, dst = _place(s, best.clamp(max=cap - 1))[real], _place(s, slot.expand_as(best).clamp(max=cap - 1))[real]
    for_all = lambda x: x.view(-1, c["d"])  # noqa: E731
    for_all(s["K"])[dst] = for_all(s["K"])[src]
    for_all(s["V"])[dst] = for_all(s["V"])[src]
    s["acc_out"].copy_(s["acc"] * (j >= L))
    s["acc_out"][:, :min(cap, c["budget"])] += (s["acc"].gather(1, best.clamp(max=cap - 1)) * real)[:, :cap]
    s["len_out"].copy_(left[:, 0])
    s["kept"].copy_(torch.where(real, best.int(), s["kept"]))
    return [s["K"], s["V"], s["acc_out"], s["len_out"], s["kept"]]


def run(state):
    s, c = state, state["c"]
    if not own:
        return {"append": _plain_append, "decode": _plain_decode, "prefill": _plain_prefill, "evict": _plain_evict}[c["op"]](s)
    x = s["ctx"]
    if c["op"] == "append":
        x.cache_append(s["k_new"], s["v_new"], s["new"], s["len"], s["K"], s["V"])
        return [s["K"], s["V"]]
    if c["op"] == "decode":
        x.cache_decode(s["q"], s["K"], s["V"], s["len"], c["window"], c["first"], s["out"], s["acc"], s["ws"])
    elif c["op"] == "prefill":
        x.cache_prefill(s["q"], s["new"], s["K"], s["V"], s["len"], c["window"], c["first"], s["out"], s["acc"], s["ws"])
    else:
        x.cache_evict(s["K"], s["V"], s["acc"], s["len"], c["budget"], c["first"], c["last"], s["acc_out"], s["len_out"], s["kept"])
        return [s["K"], s["V"], s["acc_out"], s["len_out"], s["kept"]]
    return [s["out"], s["acc"]] if c["weights"] else [s["out"]]


# ------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits, cache by cache
# ------------------------------------------------------------------------------------------------------------------
def _exact_cache(s, i, which, rows):
    """Rows `rows` of cache i in 64 bits."""
    c = s["c"]
    if s["table"] is None:
        return s[which][i, rows].double()
    return s[which][s["table"][i, rows // c["block"]].long(), rows % c["block"]].double()


def _exact_attention(s):
    c = s["c"]
    decode = c["op"] == "decode"
    out = s["out"].double()
    acc = s["acc"].double() if c["weights"] else None
    lens, new = s["len"].tolist(), s["new"].tolist()
    for i, L in enumerate(lens):
        count = 1 if decode else new[i]
        for r0 in range(0, count, 512):
            at = torch.arange(L - count + r0, L - count + min(count, r0 + 512), device="cuda")      # positions of these queries
            end, begin = int(at[-1]) + 1, 0 if not c["window"] else max(0, int(at[0]) - c["window"] + 1)
            head = torch.arange(0, min(c["first"], begin), device="cuda")
            j = torch.cat([head, torch.arange(begin, end, device="cuda")])
            q = (s["q"][i:i + 1] if decode else s["q"][i, r0:r0 + len(at)]).double()                # [m][g][d]
            x = torch.einsum("mgd,jd->gmj", q, _exact_cache(s, i, "K", j)) / math.sqrt(c["d"])
            hidden = j[None, :] > at[:, None]
            if c["window"]:
                hidden |= (at[:, None] - j[None, :] >= c["window"]) & (j[None, :] >= c["first"])
            p = torch.softmax(x.masked_fill(hidden[None], -math.inf), dim=-1)
            o = torch.einsum("gmj,jd->mgd", p, _exact_cache(s, i, "V", j))
            if decode:
                out[i] = o[0]
            else:
                out[i, r0:r0 + len(at)] = o
            if acc is not None:
                acc[i, j] += p.sum((0, 1))
    return [out, acc] if acc is not None else [out]


def exact(case, seed):
    c = case
    if c["op"] not in ("decode", "prefill"):
        # rows are moved and not computed: copies and whole numbers, held to the plain form bit by bit
        return None
    if 4.0 * c["seqs"] * c["heads"] * c["g"] * c["d"] * c["q"] * c["hi"] > 2e13:
        return None
    return _exact_attention(prepare(case, seed))
