"""Work on sequences that have pages and a beginning in common: pages are taken and given back, sequences fork, pools are compacted and
copied, and tokens attend to a beginning that many sequences share, call by call.

A case is one pass through an operator at one size.  An instance is one (layer, batch, KV head) triple; the instances of a sequence share
its length.  A page holds `block` rows of K and V; an instance's row of the block table names its pages, and refs counts how often the
table names each page.  The kinds ("op"):

  resize   tables are brought in line with lengths: pages behind an instance's rows are given back, missing ones are taken, and shared
           ones that are about to be written are replaced by copies (Context.pages_resize).  A pass gives back the rows of a step's (or
           chunk's) tokens and takes pages for new ones, as where drafted tokens are refused
  fork     every instance goes on from another one or itself: full pages are shared, a page that is not full is copied (Context.pages_fork)
  compact  the pages in use move to the front of the pool (Context.pages_compact).  A pass begins with the same scattered pages
  copy     listed pages go to other places, of another pool (Context.pages_copy)
  decode   one new token per sequence; groups of sequences have their first rows in common (Context.cache_decode_shared)
  prefill  several new tokens per sequence, the same (Context.cache_prefill_shared)

run() has each of them in its plain form, in 32 bits, and, where `own` is set, as the library's calls.
"""
import math

import torch

own = False

# prompts x seqs sequences of `heads` instances.  plo .. phi: rows that the sequences of a prompt have in common; lo .. hi: rows of a sequence's
# own behind them, the newest q tokens' included.  alone: so many of 8 sequences share nothing.
_BASE = {"op": "decode", "prompts": 1, "seqs": 4, "heads": 8, "g": 4, "d": 128, "block": 16, "dtype": "bf16", "paged": True, "plo": 2000, "phi": 2000,
         "lo": 1, "hi": 100, "q": 1, "window": 0, "first": 0, "alone": 0, "fill": 0.5, "beams": False}


def _case(name, **kw):
    return dict(_BASE, name=name, **kw)


def listed():
    return [
        # A decode step of 4 samples of one prompt in one layer, with three drafted tokens of which some were refused: latency.
        _case("resize_step", op="resize", lo=20, hi=60, q=4),
        # Chunks of prompts of 32 sequences in two layers' pool: many pages at a time.
        _case("resize_chunks", op="resize", prompts=32, seqs=1, heads=16, block=16, plo=100, phi=4100, lo=2050, hi=4100, q=2048),
        # One prompt becomes four samples: their tables name its pages, the last one is copied.
        _case("fork_samples", op="fork", seqs=4, plo=2041, phi=2041, lo=0, hi=0),
        # A step of beam search: 16 prompts with 4 beams each go on from the beams that were chosen.
        _case("fork_beams", op="fork", prompts=16, seqs=4, plo=900, phi=7900, lo=30, hi=300, beams=True),
        # A small pool, most of it in use.
        _case("compact_small", op="compact", prompts=4, seqs=1, plo=0, phi=0, lo=200, hi=2030, fill=0.9),
        # After many sequences have ended: a pool of a third in use gives its end back.
        _case("compact_pool", op="compact", prompts=40, seqs=1, plo=0, phi=0, lo=300, hi=8190, fill=0.35),
        # The pages of one sequence of one layer leave for another pool, as where it has to wait.
        _case("copy_one_seq", op="copy", seqs=1, plo=0, phi=0, lo=2041, hi=2041),
        # The same for 16 sequences of different lengths.
        _case("copy_seqs", op="copy", prompts=16, seqs=1, plo=0, phi=0, lo=700, hi=16380),
        # Four samples of one prompt, one layer: the latency of a decode step.
        _case("decode_samples", plo=2041, phi=2041, lo=1, hi=200),
        # 64 sequences behind one long system prompt, of their own lengths.
        _case("decode_system", seqs=64, plo=8190, phi=8190, lo=40, hi=2050),
        # 16 sequences of two prompts with five drafted tokens each.
        _case("prefill_drafts", op="prefill", prompts=2, seqs=8, plo=4000, phi=8190, lo=30, hi=700, q=5),
        # 8 questions of up to 100 tokens behind one document.
        _case("prefill_questions", op="prefill", seqs=8, plo=6000, phi=6000, lo=101, hi=101, q=100),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(_BASE, op=rng.choice(["resize", "fork", "compact", "copy", "decode", "decode", "decode", "prefill", "prefill"]))
    c["heads"] = rng.choice([1, 2, 8, 8, 8, 16])
    c["g"] = rng.choice([1, 2, 4, 4, 4, 8])
    c["d"] = rng.choice([64, 128, 128])
    c["block"] = rng.choice([8, 16, 16, 32, 64])
    c["dtype"] = rng.choice(["f32", "bf16", "bf16", "bf16", "bf16"])
    size = c["d"] * (2 if c["dtype"] == "bf16" else 4)
    c["phi"] = _log_int(rng, 8, 8000)
    c["plo"] = max(1, int(c["phi"] * rng.choice([0.1, 0.7, 1.0])))
    c["hi"] = _log_int(rng, 2, 2000)
    c["lo"] = max(1, int(c["hi"] * rng.choice([0.02, 0.5, 1.0])))
    c["alone"] = rng.choice([0, 0, 0, 1, 4])
    rows = c["phi"] + c["hi"]
    if c["op"] in ("decode", "prefill"):
        most = 1.0e9 / (rows * size)                          # instances: bounded by the bytes of K if nothing were shared ...
        c["paged"] = rng.random() < 0.8
        c["window"] = rng.choice([0, 0, 0, max(1, int(rows * rng.uniform(0.05, 0.9)))])
        c["first"] = rng.choice([0, 1, 4, 37]) if c["window"] else 0
        if c["op"] == "prefill":                              # ... and by the scores of the plain form
            c["q"] = min(c["hi"], _log_int(rng, 1, 200))
            most = min(most, 2.5e8 / (c["q"] * c["g"] * rows))
    else:
        most = 0.4e9 / (rows * size)
        if c["op"] == "resize":
            c["q"] = min(rows, _log_int(rng, 1, 1000))
        c["beams"] = rng.random() < 0.7
        c["fill"] = rng.uniform(0.1, 0.95)
    n = max(2, min(512, _log_int(rng, 2, max(2.0, most / c["heads"]))))
    c["seqs"] = max(1, min(n, _log_int(rng, 1, 64)))
    c["prompts"] = max(1, n // c["seqs"])
    return c


# ------------------------------------------------------------------------------------------------------------------
# Sizes, from the case alone; the seed only says which sequence has which length
# ------------------------------------------------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n whole numbers from lo to hi, even over their logarithm, hi among them."""
    if n == 1 or hi < 1:
        return [hi] * n
    lo = max(lo, 1)
    at = [((k * 0.6180339887498949) % 1.0) for k in range(n - 1)]
    return [hi] + [max(1, min(hi, int(round(lo * (hi / lo) ** u)))) for u in at]


def _sizes(c):
    """Of every sequence: its prompt, the rows that it has in common with that (0: alone), its length and its new tokens.  The sequences of a
    prompt lie `prompts` apart."""
    n = c["prompts"] * c["seqs"]
    first, own_rows, new = _spread(c["prompts"], c["plo"], c["phi"]), _spread(n, c["lo"], c["hi"]), _spread(n, max(1, (2 * c["q"]) // 3), c["q"])
    out = []
    for s in range(n):
        p = s % c["prompts"]
        mine = own_rows[p] if c["op"] == "fork" else own_rows[s]             # beams have one length
        alone = (s // c["prompts"] * 5 + p) % 8 < c["alone"]
        # (a table may go back into rows in common, whose pages are then copied; attention's new tokens lie behind them)
        out.append((p, 0 if alone else first[p], first[p] + mine, min(new[s], first[p] + mine if c["op"] == "resize" else max(1, mine))))
    return out


def _groups(sizes):
    """(prompt, rows in common, lengths and new tokens of its sequences that share); a sequence that shares nothing is a group of its own."""
    got = {}
    for i, (p, shared, n, k) in enumerate(sizes):
        got.setdefault((p, 0) if shared else (p, 1 + i), [shared, []])[1].append((n, k))
    return list(got.values())


def _seen(c, p):
    """Rows that a query at position p sees."""
    if not c["window"]:
        return p + 1
    return min(p + 1, c["window"]) + max(0, min(c["first"], p + 1 - c["window"]))


def _pages(c, n):
    return -(-n // c["block"])


def work(case):
    c = case
    sizes = _sizes(c)
    row = c["d"] * (2 if c["dtype"] == "bf16" else 4)
    h, g, b, n = c["heads"], c["g"], c["block"], len(sizes)
    if c["op"] == "resize":
        changed = sum(_pages(c, L) - _pages(c, L - k) for _, _, L, k in sizes)
        return {"bytes": h * (16 * changed + 16 * n) + 16, "flops": 0}
    if c["op"] == "fork":
        go_on = [(i, p) for i, p in enumerate(_parents(c)) if p != i and p >= 0]
        moved = sum(2 * 4 * _pages(c, sizes[p][2]) + 4 * row * (sizes[p][2] % b) for i, p in go_on)
        return {"bytes": h * (moved + 12 * n) + 8, "flops": 0}
    if c["op"] == "compact":
        live = h * sum(_pages(c, L) for _, _, L, _ in sizes)
        total = _pool(c, live)
        moved = live * (total - live) // total                # of pages that lie anywhere, as many lie behind the first `live`
        return {"bytes": 4 * row * b * moved + 8 * live + 8 * total, "flops": 0}
    if c["op"] == "copy":
        pages = h * sum(_pages(c, L) for _, _, L, _ in sizes)
        return {"bytes": pages * (4 * row * b + 8), "flops": 0}
    rows = pairs = queries = 0
    for shared, members in _groups(sizes):
        lowest = min(L - k for L, k in members)               # position of the first query
        rows += shared if not c["window"] else min(shared, max(0, shared - (lowest + 1 - c["window"])) + c["first"])
        for L, k in members:
            queries += k
            rows += L - shared if not c["window"] else min(L - shared, c["window"] + k - 1)
            pairs += sum(_seen(c, L - k + r) for r in range(k))
    out = 4 if c["op"] == "decode" else row // c["d"]
    tables = 4 * rows / b if c["paged"] else 0
    return {"bytes": h * (2 * row * rows + tables + queries * g * (row + out * c["d"]) + 16 * n), "flops": 4 * h * g * c["d"] * pairs}


# ------------------------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------------------------
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _generator(seed, what):
    gen = torch.Generator(device="cuda")
    gen.manual_seed((int(seed) * 1000003 + what * 7919 + 4321) % (1 << 62))
    return gen


def _normal(shape, c, seed, what, scale=1.0):
    x = torch.empty(shape, dtype=_dtype(c), device="cuda").normal_(generator=_generator(seed, what))
    return x if scale == 1.0 else x.mul_(scale)


def _pool(c, live):
    """Pages of a pool that is to be compacted."""
    return max(live, int(round(live / c["fill"])))


def _parents(c):
    """The sequence that every sequence goes on from; -1: none, it ends.  Samples go on from their prompt's first sequence; of beams, some are
    chosen several times, some not at all, and one in eight of those ends."""
    n, p = c["prompts"] * c["seqs"], c["prompts"]
    if not c["beams"]:
        return [s % p for s in range(n)]
    parent = [s % p + p * (((s // p) * 7 + (s % p) * 3) // 4 * 2 % c["seqs"]) for s in range(n)]
    chosen = set(parent)
    return [-1 if s not in chosen and (s * 5) % 8 == 3 else parent[s] for s in range(n)]


def _heads(c, v):
    """Values of the sequences as those of their instances, int32."""
    return torch.tensor([x for x in v for _ in range(c["heads"])], dtype=torch.int32, device="cuda")


def _table(c, gen, sizes, cap, spare, share=True):
    """A table whose pages lie anywhere in a pool, and the pool's pages: full pages of the rows in common are named by every sequence of the
    prompt (the first sharing one's), the others are an instance's own."""
    h, nb, n = c["heads"], cap // c["block"], len(sizes)
    names, first, count = torch.full((n, nb), -1, dtype=torch.int64), {}, 0
    for s, (p, shared, L, _) in enumerate(sizes):
        common = shared // c["block"] if share else 0
        at = 0
        if common:
            if p in first:
                names[s, :common] = names[first[p], :common]
                at = common
            else:
                first[p] = s
        more = _pages(c, L) - at
        names[s, at:at + more] = torch.arange(count, count + more)
        count += more
    names = names.to("cuda")[:, None, :]
    head = torch.arange(h, device="cuda")[None, :, None]
    names = torch.where(names >= 0, names * h + head, -1).view(n * h, nb)    # pages of a row of heads lie together, before they are mixed
    live = count * h
    pool = _pool(c, live) if c["op"] == "compact" else live + spare
    mixed = torch.randperm(pool, generator=gen, device="cuda")
    return torch.where(names >= 0, mixed[names.clamp(min=0)], -1).to(torch.int32).contiguous(), pool


def _refs(table, pool):
    named = table[table >= 0].long()
    return torch.bincount(named, minlength=pool).to(torch.int32)


def prepare(case, seed):
    c = case
    sizes = _sizes(c)
    if c["op"] != "fork":                                     # which prompt's sequence has which rows goes by the seed
        p, turn = c["prompts"], int(seed) % c["seqs"]
        sizes = sizes[turn * p:] + sizes[:turn * p]
    n = len(sizes) * c["heads"]
    cap = -(-(max(L for _, _, L, _ in sizes) + 1) // 64) * 64
    b, d, gen = c["block"], c["d"], _generator(seed, 7)
    s = {"c": c, "cap": cap, "n": n, "len": _heads(c, [x[2] for x in sizes]), "new": _heads(c, [x[3] for x in sizes])}
    if c["op"] in ("decode", "prefill"):
        share = _heads(c, [x[1] for x in sizes])
        group = torch.tensor([x[0] * c["heads"] + h if x[1] else -1 for x in sizes for h in range(c["heads"])], dtype=torch.int32, device="cuda")
        s["table"], pool = _table(c, gen, sizes, cap, 1) if c["paged"] else (None, 0)
        shape = (pool, b, d) if c["paged"] else (n, cap, d)
        s["K"], s["V"] = _normal(shape, c, seed, 1), _normal(shape, c, seed, 2)
        # Rows in common that lie in pages (caches) of an instance's own hold what those of the group's first instance hold.
        first = torch.full((n,), n, dtype=torch.int64, device="cuda")
        at = torch.arange(n, device="cuda")
        key = torch.where(group >= 0, group.long(), 0)
        first = torch.where(group >= 0, torch.full_like(first, n).scatter_reduce(0, key, torch.where(group >= 0, at, n), "amin")[key], at)
        begin = (share // b * b) if c["paged"] else torch.zeros_like(share)
        width = b if c["paged"] else max(1, c["phi"])
        j = begin[:, None] + torch.arange(width, device="cuda")[None, :]
        real = (j < share[:, None]) & (first != at)[:, None]
        to, src = _place(s, j.clamp(max=cap - 1))[real], _place(s, j.clamp(max=cap - 1), first)[real]
        for x in (s["K"], s["V"]):
            x.view(-1, d)[to] = x.view(-1, d)[src]
        lead = (n, c["g"], d) if c["op"] == "decode" else (n, c["q"], c["g"], d)
        # Queries of twice the keys' size: scores spread by two, so that few rows carry most of the weight.
        s["q"] = _normal(lead, c, seed, 5, 2.0)
        s["out"] = torch.zeros(lead, dtype=torch.float32 if c["op"] == "decode" else _dtype(c), device="cuda")
        s["group"], s["shared"] = group, share
    else:
        # (pages that a pass gives back serve from the next one on)
        spare = {"resize": n * (_pages(c, c["q"]) + 2), "fork": 2 * n, "compact": 0, "copy": 3}[c["op"]]
        s["table"], pool = _table(c, gen, sizes, cap, spare, share=c["op"] != "copy")
        s["pool"] = pool
        s["K"], s["V"] = _normal((pool, b, d), c, seed, 1), _normal((pool, b, d), c, seed, 2)
        s["state"] = _refs(s["table"], pool)
        s["info"], s["info2"] = (torch.zeros((2,), dtype=torch.int32, device="cuda") for _ in range(2))
        if c["op"] == "resize":
            s["short"] = s["len"] - s["new"]
        if c["op"] == "fork":
            of = torch.arange(c["heads"], device="cuda")[None, :]
            parent = torch.tensor(_parents(c), device="cuda")[:, None]
            s["parent"] = torch.where(parent >= 0, parent * c["heads"] + of, -1).to(torch.int32).view(-1).contiguous()
        if c["op"] == "copy":
            s["src"] = s["table"][s["table"] >= 0].contiguous()
            s["dst"] = torch.randperm(s["src"].numel() + 5, generator=gen, device="cuda")[:s["src"].numel()].to(torch.int32)
            s["K2"], s["V2"] = (torch.zeros((s["src"].numel() + 5, b, d), dtype=_dtype(c), device="cuda") for _ in range(2))
    if own:
        from paper_2502_04077_amd import Context
        x = s["ctx"] = Context(n_inst=n, g=c["g"], head_dim=d, block=b, hist_len=1, t_cap=cap, k_blocks=1, n_sink=0, n_local=0, c1=4, c2=4,
                               kv_dtype=c["dtype"])
        if c["op"] in ("decode", "prefill"):
            if c["paged"]:
                x.set_block_table(s["table"], pool)
            s["plan"] = torch.zeros(x.cache_share_bytes(), dtype=torch.uint8, device="cuda")
            x.cache_share(s["group"], s["shared"], s["plan"])
            size = x.cache_shared_workspace_bytes(c["q"] if c["op"] == "prefill" else 0)
        else:
            s["state"] = torch.zeros(x.pages_state_bytes(pool) // 4, dtype=torch.int32, device="cuda")
            x.pages_count(s["table"], pool, s["state"])
            size = x.pages_workspace_bytes(pool)
        s["ws"] = torch.zeros(max(16, size), dtype=torch.uint8, device="cuda")
    if c["op"] == "compact":
        s["table0"], s["state0"] = s["table"].clone(), s["state"].clone()
    return s


# ------------------------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------------------------
def _place(s, at, of=None):
    """Rows of the pool, seen as [rows][d], at which rows `at` [n][m] of the caches lie (of: of the caches of these instances)."""
    c = s["c"]
    of = torch.arange(s["n"], device="cuda") if of is None else of
    at = at.long()
    if s["table"] is None:
        return of[:, None] * s["cap"] + at
    return s["table"].long()[of].gather(1, at // c["block"]).clamp(min=0) * c["block"] + at % c["block"]


def _rows(s, which, n_rows):
    """The first n_rows rows of every cache, in 32 bits: [n][n_rows][d]."""
    at = torch.arange(n_rows, device="cuda")[None, :].expand(s["n"], n_rows)
    return s[which].view(-1, s["c"]["d"])[_place(s, at)].float()


def _attend(s, q, pos, n_rows):
    """q [n][m][g][d] at positions pos [n][m]: outputs [n][m][g][d]."""
    c = s["c"]
    n, m, g, d = q.shape
    K, V = _rows(s, "K", n_rows), _rows(s, "V", n_rows)
    j, p = torch.arange(n_rows, device="cuda")[None, None, :], pos[:, :, None]
    hidden = j > p
    if c["window"]:
        hidden = hidden | ((j <= p - c["window"]) & (j >= c["first"]))
    w = torch.matmul(q.float().view(n, m * g, d), K.transpose(1, 2).contiguous()).view(n, m, g, n_rows)
    w = w.mul_(1.0 / math.sqrt(d)).masked_fill_(hidden[:, :, None, :], -math.inf)
    top = w.amax(-1, keepdim=True)
    w = w.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = w.sum(-1, keepdim=True)
    w = w.div_(torch.where(total == 0, 1.0, total))
    return torch.matmul(w.view(n, m * g, n_rows), V).view(n, m, g, d)


def _plain_decode(s):
    s["out"].copy_(_attend(s, s["q"][:, None], s["len"][:, None] - 1, s["c"]["phi"] + s["c"]["hi"])[:, 0])
    return [s["out"]]


def _plain_prefill(s):
    c = s["c"]
    r = torch.arange(c["q"], device="cuda")[None, :]
    good = r < s["new"][:, None]
    out = _attend(s, s["q"], (s["len"] - s["new"])[:, None] + r, c["phi"] + c["hi"])
    s["out"].copy_(torch.where(good[:, :, None, None], out.to(s["out"].dtype), s["out"]))
    return [s["out"]]


def _count(refs, entries, by):
    """refs += by for every entry that names a page."""
    real = (entries >= 0) & (entries < refs.shape[0])
    refs.index_add_(0, entries[real].long(), torch.full_like(entries[real], by))


def _move(s, src, dst, rows):
    """The first rows[i] rows of page src[i] go to page dst[i]."""
    if not src.numel():
        return
    r = torch.arange(s["c"]["block"], device="cuda")[None, :]
    real = r < rows[:, None]
    b = s["c"]["block"]
    for x in (s["K"].view(-1, s["c"]["d"]), s["V"].view(-1, s["c"]["d"])):
        x[(dst.long()[:, None] * b + r)[real]] = x[(src.long()[:, None] * b + r)[real]]


def _take(refs, need):
    """A free page for every place that needs one, the lowest first, in the places' order; None where there are too few, and how many are lacking."""
    free = (refs == 0).nonzero()[:, 0].to(torch.int32)
    lacking = (need.sum() - free.shape[0]).clamp(min=0).to(torch.int32)
    if int(lacking) > 0:
        return None, lacking
    rank = need.view(-1).cumsum(0).view(need.shape) - 1
    if not free.numel():
        return torch.full_like(rank, -1, dtype=torch.int32), lacking
    return free[rank.clamp(0, free.shape[0] - 1)], lacking


def _resize(s, length, new, info):
    c, table, refs, b = s["c"], s["table"], s["state"][:s["pool"]], s["c"]["block"]
    k = torch.arange(table.shape[1], device="cuda")[None, :]
    want = ((length + b - 1) // b)[:, None]
    start = (length - new)[:, None]                           # the first row to be written
    named = (table >= 0) & (table < s["pool"])
    shared = named & (refs[table.clamp(0, s["pool"] - 1).long()] > 1)
    copied = shared & (k < want) & (k >= start // b) & (new > 0)[:, None]
    need = copied | (~named & (k < want))
    page, lacking = _take(refs, need)
    if page is not None:
        old = table.clone()
        _count(refs, old[named & ((k >= want) | copied)], -1)
        table.masked_fill_(k >= want, -1)
        table.copy_(torch.where(need, page, table))
        _count(refs, table[need], 1)
        keep = (start - k * b).clamp(0, b)
        _move(s, old[copied], table[copied], keep[copied])
    info.copy_(torch.stack([(refs == 0).sum().to(torch.int32), lacking]))


def _plain_resize(s):
    _resize(s, s["short"], torch.zeros_like(s["new"]), s["info"])
    _resize(s, s["len"], s["new"], s["info2"])
    return [s["table"], s["state"][:s["pool"]], s["info"], s["info2"], s["K"], s["V"]]


def _plain_fork(s):
    c, table, refs, b, n = s["c"], s["table"], s["state"][:s["pool"]], s["c"]["block"], s["n"]
    at, k = torch.arange(n, device="cuda"), torch.arange(s["table"].shape[1], device="cuda")[None, :]
    parent = s["parent"].long()
    some = (parent >= 0) & (parent < n)
    src = torch.where(some, parent, at)
    stays = src == at
    # The lowest instance that goes on from one that does not go on itself takes over its page that is not full.
    lowest = torch.full((n,), n, device="cuda").scatter_reduce(0, src, torch.where(some, at, n), "amin")
    heir = some & ~stays & (at == lowest[src]) & (parent[src] != src)
    length = torch.where(some, s["len"][src], 0)
    full, rest = (length // b)[:, None], length % b
    goes = (some & ~stays)[:, None]
    table2 = torch.where(k < full + (heir & (rest > 0))[:, None], table[src], -1)
    last = (k == full) & (rest > 0)[:, None] & goes & ~heir[:, None] & (table[src] >= 0) & (table[src] < s["pool"])
    page, lacking = _take(refs, last)
    if page is not None:
        changed = ~(some & stays)
        table2 = torch.where(changed[:, None], torch.where(last, page, table2), table)
        _count(refs, table2[changed], 1)
        _count(refs, table[changed], -1)
        _move(s, table[src][last], page[last], rest[:, None].expand_as(last)[last])
        table.copy_(table2)
        s["len"].copy_(length)
    s["info"].copy_(torch.stack([(refs == 0).sum().to(torch.int32), lacking]))
    return [table, refs, s["len"], s["info"], s["K"], s["V"]]


def _plain_compact(s):
    s["table"].copy_(s["table0"])
    s["state"].copy_(s["state0"])
    table, refs = s["table"], s["state"][:s["pool"]]
    at = torch.arange(s["pool"], device="cuda")
    used = refs > 0
    live = used.sum()
    src, dst = (used & (at >= live)).nonzero()[:, 0], (~used & (at < live)).nonzero()[:, 0]
    to = at.clone()
    to[src] = dst
    table.copy_(torch.where((table >= 0) & (table < s["pool"]), to[table.clamp(0, s["pool"] - 1).long()].to(torch.int32), table))
    refs[dst] = refs[src]
    refs[src] = 0
    s["K"][dst] = s["K"][src]
    s["V"][dst] = s["V"][src]
    s["info"].copy_(torch.stack([s["pool"] - live, torch.tensor(src.shape[0], device="cuda")]))
    return [table, refs, s["info"], s["K"], s["V"]]


def _plain_copy(s):
    s["K2"][s["dst"].long()] = s["K"][s["src"].long()]
    s["V2"][s["dst"].long()] = s["V"][s["src"].long()]
    return [s["K2"], s["V2"]]


def run(state):
    s, c = state, state["c"]
    if not own:
        return {"resize": _plain_resize, "fork": _plain_fork, "compact": _plain_compact, "copy": _plain_copy, "decode": _plain_decode,
                "prefill": _plain_prefill}[c["op"]](s)
    x = s["ctx"]
    if c["op"] == "resize":
        x.pages_resize(s["K"], s["V"], s["table"], s["state"], s["short"], None, 0, s["info"], s["ws"])
        x.pages_resize(s["K"], s["V"], s["table"], s["state"], s["len"], s["new"], c["q"], s["info2"], s["ws"])
        return [s["table"], s["state"][:s["pool"]], s["info"], s["info2"], s["K"], s["V"]]
    if c["op"] == "fork":
        x.pages_fork(s["K"], s["V"], s["table"], s["state"], s["parent"], s["len"], s["len"], s["info"], s["ws"])
        return [s["table"], s["state"][:s["pool"]], s["len"], s["info"], s["K"], s["V"]]
    if c["op"] == "compact":
        s["table"].copy_(s["table0"])
        s["state"].copy_(s["state0"])
        x.pages_compact(s["K"], s["V"], s["table"], s["state"], s["info"], s["ws"])
        return [s["table"], s["state"][:s["pool"]], s["info"], s["K"], s["V"]]
    if c["op"] == "copy":
        x.pages_copy(s["K"], s["V"], s["src"], s["K2"], s["V2"], s["dst"])
        return [s["K2"], s["V2"]]
    if c["op"] == "decode":
        x.cache_decode_shared(s["q"], s["K"], s["V"], s["len"], s["plan"], c["window"], c["first"], s["out"], s["ws"])
    else:
        x.cache_prefill_shared(s["q"], s["new"], s["K"], s["V"], s["len"], s["plan"], c["window"], c["first"], s["out"], s["ws"])
    return [s["out"]]


# ------------------------------------------------------------------------------------------------------------------
# The definition of the attention in 64 bits, cache by cache
# ------------------------------------------------------------------------------------------------------------------
def _exact_rows(s, i, which, rows):
    """Rows `rows` of cache i in 64 bits."""
    if s["table"] is None:
        return s[which][i, rows].double()
    b = s["c"]["block"]
    return s[which][s["table"][i, rows // b].long(), rows % b].double()


def exact(case, seed):
    c = case
    if c["op"] not in ("decode", "prefill"):
        # pages are moved and counted, nothing is computed: copies and whole numbers, held to the plain form bit by bit
        return None
    s = prepare(case, seed)
    decode = c["op"] == "decode"
    out = s["out"].double()
    for i, (L, k) in enumerate(zip(s["len"].tolist(), s["new"].tolist())):
        count = 1 if decode else k
        at = torch.arange(L - count, L, device="cuda")        # positions of the queries
        low = 0 if not c["window"] else max(0, L - count - c["window"] + 1)
        j = torch.cat([torch.arange(0, min(c["first"], low), device="cuda"), torch.arange(low, L, device="cuda")])
        q = (s["q"][i:i + 1] if decode else s["q"][i, :count]).double()       # [m][g][d]
        x = torch.einsum("mgd,jd->gmj", q, _exact_rows(s, i, "K", j)) / math.sqrt(c["d"])
        seen = j[None, :] <= at[:, None]
        if c["window"]:
            seen &= (at[:, None] - j[None, :] < c["window"]) | (j[None, :] < c["first"])
        w = torch.softmax(torch.where(seen[None], x, -math.inf), dim=-1)
        o = torch.einsum("gmj,jd->mgd", w, _exact_rows(s, i, "V", j))
        if decode:
            out[i] = o[0]
        else:
            out[i, :count] = o
    return [out]
