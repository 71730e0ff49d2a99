"""Operators of one serving step around the low-bit cache, over the sizes a serving program meets, for measuring them.

A step of many requests first finds room for its new rows in the paged cache, turns queries and keys to their positions, adds each
request's own low-rank weights to a shared projection, and at the end draws a token from each row's logits:

  pages      page tables, rows and slot maps from the lengths that the requests want (sl_kv8_pages_resize)
  rope       rotary positions of rows of queries and keys (sl_rope_rows)
  adapters   y = base + scale (x A^T) B^T with an adapter for each row (sl_adapters_forward)
  sample     temperature, top-k, top-p, min-p and a draw from a given uniform number (sl_sample_filtered)

`own` chooses between the plain formulas below and the library's kernels.  Definitions:

  pages      a sequence of len slots holds ceil(len / page_slots) pages.  Sequences that want less release their last pages.  Then, in
             order, each that wants more takes pages, unless too few pages or rows are left for all of it: then it stays.  The i-th page
             taken is the i-th released; beyond those, pages come from the top of the stack of free ones, or go on top of it.
             Every new slot is a row: its place, its length (place + 1), its sequence and its slot in the pool
  rope       a pair (a, b) -> (a cos t - b sin t, a sin t + b cos t) amplitude, t = position * frequency; pairs are (j, j + rot / 2) or
             (2 j, 2 j + 1); numbers behind the first rot of a head stay
  adapters   as above; base may come in several partial sums; rows without an adapter get base alone
  sample     weights W = rint(2^44 exp((z - max z) / temperature)), as whole numbers; NaN and -infinity are never drawn.  Tokens in
             descending order of z, ties to the lower id: the first top_k of them; of these the fewest that hold top_p of their weight;
             of these the ones with W >= min_p 2^44, at least one.  The token is the lowest id whose running weight among the kept exceeds u times
             their sum.  Temperature 0 takes the first of the order
"""
import math

import torch

own = False
DEV = "cuda:0"
LLADA_D, LLADA_HEADS, LLADA_HEAD, LLADA_FF, LLADA_VOCAB = 4096, 32, 128, 12288, 126464     # the LLaDA-8B-shaped model
TINY_D, TINY_HEADS, TINY_HEAD, TINY_FF, TINY_VOCAB = 256, 4, 64, 688, 1024                 # the tiny fp32 model
UNIT = 2.0 ** 44
LISTS = ("lens", "want")


# ---- the cases ------------------------------------------------------------------------------------
def listed():
    return [
        # three sequences of a small cache, one row more each: launch and latency
        {"name": "pages_tiny_b3", "kind": "pages", "page": 16, "lens": "31 32 5", "want": "32 33 6", "spare": 4, "rows": 3, "max_pages": 8},
        # a full batch in decoding: a row more each, some crossing into a new page, some done, some just begun
        {"name": "pages_255_decoding", "kind": "pages", "page": 64, "lens": _spread(255, 7, 1, 4000), "want": _decoding(255, 7, 1, 4000), "spare": 300,
         "rows": 4096, "max_pages": 64},
        # prompts of a batch of 64 arrive as older requests end: the rows of a long prefill, small pages, and not room for all of them
        {"name": "pages_64_prompts", "kind": "pages", "page": 16, "lens": _spread(64, 3, 2000, 8000), "want": _prompts(64, 5, 6000, 16000), "spare": 60,
         "rows": 262144, "max_pages": 1024},
        # three rows of the tiny model: launch and latency
        {"name": "rope_tiny_m3", "kind": "rope", "rows": 3, "heads": TINY_HEADS, "kv_heads": TINY_HEADS, "d": TINY_HEAD, "rot": TINY_HEAD, "interleaved": False,
         "in": "fp32", "out": "fp32", "most": 128, "scaling": "plain"},
        # a late step of a batch of eight with long sequences: fp32 from a product, bf16 for the cache, half of the head turned, neighbours in pairs
        {"name": "rope_m137_long", "kind": "rope", "rows": 137, "heads": LLADA_HEADS, "kv_heads": 8, "d": LLADA_HEAD, "rot": 64, "interleaved": True,
         "in": "fp32", "out": "bf16", "most": 1000000, "scaling": "turns"},
        # the first step of a batch of eight ragged sequences, as columns of the fused projection
        {"name": "rope_8_prompts", "kind": "rope", "rows": 5533, "heads": LLADA_HEADS, "kv_heads": LLADA_HEADS, "d": LLADA_HEAD, "rot": LLADA_HEAD,
         "interleaved": False, "in": "bf16", "out": "bf16", "most": 1024, "scaling": "plain"},
        # one row of one request beside the Out projection: launch and latency
        {"name": "adapters_out_m1", "kind": "adapters", "rows": 1, "n": LLADA_D, "k": LLADA_D, "slots": 4, "max_rank": 16, "run": 1, "splits": 1, "out": "fp32"},
        # 64 requests of one row, an adapter each, beside the fused Q|K|V projection
        {"name": "adapters_qkv_m64", "kind": "adapters", "rows": 64, "n": 3 * LLADA_D, "k": LLADA_D, "slots": 64, "max_rank": 16, "run": 1, "splits": 1,
         "out": "bf16"},
        # the prompts of some requests: long runs of rows with one adapter, higher ranks, beside the down projection in two partial sums
        {"name": "adapters_down_m1100", "kind": "adapters", "rows": 1100, "n": LLADA_D, "k": LLADA_FF, "slots": 12, "max_rank": 64, "run": 150, "splits": 2,
         "out": "bf16"},
        # a row of the tiny model: launch and latency
        {"name": "sample_tiny_m3", "kind": "sample", "rows": 3, "vocab": TINY_VOCAB, "dtype": "fp32", "top_k": 3, "top_p": False, "min_p": False, "mapped": False},
        # the masked rows of a block: the usual filters together
        {"name": "sample_m64_top_k_p", "kind": "sample", "rows": 64, "vocab": LLADA_VOCAB, "dtype": "bf16", "top_k": 50, "top_p": True, "min_p": False,
         "mapped": True},
        # every row of a long prompt's worth: top-p and min-p over the whole vocabulary
        {"name": "sample_m1024_top_p", "kind": "sample", "rows": 1024, "vocab": LLADA_VOCAB, "dtype": "bf16", "top_k": 0, "top_p": True, "min_p": True,
         "mapped": False},
    ]


def _numbers(count, salt):
    """Some whole numbers, always the same: what a list of lengths is made of."""
    x, out = salt * 7919 + 12345, []
    for _ in range(count):
        x = (x * 1103515245 + 12345) % (1 << 31)
        out.append(x >> 8)
    return out


def _spread(count, salt, lo, hi):
    return " ".join(str(lo + x % (hi - lo + 1)) for x in _numbers(count, salt))


def _decoding(count, salt, lo, hi):
    """One slot more each; every sixteenth has ended, every twentieth has just got a prompt of 37 more."""
    return " ".join(str(0 if i % 16 == 9 else lo + x % (hi - lo + 1) + (37 if i % 20 == 3 else 1)) for i, x in enumerate(_numbers(count, salt)))


def _prompts(count, salt, lo, hi):
    """Half of the sequences end, the others have grown to what their new prompts need."""
    return " ".join(str(0 if i % 2 else lo + x % (hi - lo + 1)) for i, x in enumerate(_numbers(count, salt)))


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _opened(c):
    """The case with its lists (a number a sequence, as text) as lists."""
    return {n: [int(x) for x in v.split()] if n in LISTS and isinstance(v, str) else v for n, v in c.items()}


def _cost(c):
    """A rough time, to keep drawn cases below the largest listed one of their kind."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 4e14


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    kind = rng.choice(["pages", "rope", "adapters", "adapters", "sample", "sample"])
    while True:
        if kind == "pages":
            page = rng.choice([16, 32, 64, 128, 256])
            lens = [rng.choice([0, _log_int(rng, 1, 16000)]) for _ in range(_log_int(rng, 1, 255))]
            want = [rng.choice([n + 1, n + 1, n + 1, n, -1, 0, n // 2, n + _log_int(rng, 1, 4000)]) for n in lens]
            held = max(-(-max(n, w) // page) for n, w in zip(lens, want))
            c = {"kind": kind, "page": page, "lens": lens, "want": want, "spare": _log_int(rng, 1, 2000), "rows": _log_int(rng, 1, 262144),
                 "max_pages": max(1, held) + rng.choice([0, 0, 1, 30])}
        elif kind == "rope":
            d = rng.choice([32, 64, 80, 96, 128, 128, 128, 256])
            kv = rng.choice([1, 2, 4, 8, 32])
            c = {"kind": kind, "rows": _log_int(rng, 1, 8192), "heads": kv * (rng.choice([1, 2, 4, 8]) if kv < 32 else 1), "kv_heads": kv, "d": d,
                 "rot": rng.choice([d, d, d // 2, d // 4]), "interleaved": rng.random() < 0.5, "in": rng.choice(["bf16", "fp32"]),
                 "out": rng.choice(["bf16", "bf16", "fp32"]), "most": _log_int(rng, 100, 1000000), "scaling": rng.choice(["plain", "linear", "base", "turns"])}
        elif kind == "adapters":
            c = {"kind": kind, "rows": _log_int(rng, 1, 2048), "n": rng.choice([_log_int(rng, 64, 2 * LLADA_FF), 8 * _log_int(rng, 8, LLADA_FF // 4), LLADA_D]),
                 "k": rng.choice([8 * _log_int(rng, 8, LLADA_FF // 8), TINY_D, TINY_FF, LLADA_D, LLADA_FF]), "slots": _log_int(rng, 1, 64),
                 "max_rank": rng.choice([4, 8, 16, 16, 32, 64, 128]), "run": rng.choice([1, 1, _log_int(rng, 1, 300)]), "splits": rng.choice([1, 1, 1, 2, 4]),
                 "out": rng.choice(["bf16", "bf16", "fp32"])}
        else:
            vocab = rng.choice([_log_int(rng, 50, LLADA_VOCAB), TINY_VOCAB, LLADA_VOCAB, LLADA_VOCAB])
            c = {"kind": kind, "rows": _log_int(rng, 1, 1024), "vocab": vocab, "dtype": rng.choice(["bf16", "bf16", "fp32"]),
                 "top_k": rng.choice([0, 0, min(vocab, rng.choice([1, 20, 50, 1000, 20000]))]), "top_p": rng.random() < 0.6, "min_p": rng.random() < 0.4,
                 "mapped": rng.random() < 0.3}
        if _cost(c) <= most[kind]:
            return {n: " ".join(map(str, v)) if isinstance(v, list) else v for n, v in c.items()}


def work(c):
    """Each input once and each output once."""
    c = _opened(c)
    if c["kind"] == "pages":
        _, _, _, new, _ = _resized(c)
        rows = sum(max(0, n - o) for n, o in zip(new, c["lens"]))
        entries = len(c["lens"]) * c["max_pages"]
        return {"bytes": 4.0 * (2 * entries + 2 * _pool(c) + 4 * len(c["lens"])) + rows * 20.0, "flops": 2.0 * entries}
    ts = {n: 2 if c.get(n) == "bf16" else 4 for n in ("in", "out", "dtype")}
    if c["kind"] == "rope":
        numbers = c["rows"] * (c["heads"] + c["kv_heads"]) * float(c["d"])
        return {"bytes": numbers * (ts["in"] + ts["out"]) + 4.0 * c["rows"], "flops": 3.0 * numbers * c["rot"] / c["d"]}
    if c["kind"] == "adapters":
        which, ranks = _adapter_of_rows(c, 0), _ranks(c)
        seen = sum(ranks[a] for a in set(which) if a >= 0)
        used = sum(ranks[a] for a in which if a >= 0)
        return {"bytes": 2.0 * seen * (c["n"] + c["k"]) + c["rows"] * (2.0 * c["k"] + c["n"] * (4.0 * c["splits"] + ts["out"])),
                "flops": 2.0 * used * (c["n"] + c["k"])}
    return {"bytes": c["rows"] * (c["vocab"] * float(ts["dtype"]) + 32), "flops": c["rows"] * c["vocab"] * (4.0 if c["top_k"] else 24.0)}


# ---- inputs, from the seed alone --------------------------------------------------------------------
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + what) % (1 << 62))


def _host(seed, what):
    return torch.Generator().manual_seed((int(seed) * 1000003 + what) % (1 << 62))


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=gen).to(dtype)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _held(c, n):
    return -(-n // c["page"])


def _pool(c):
    return sum(_held(c, n) for n in c["lens"]) + c["spare"]


def _page_inputs(c, seed):
    """A pool in use: pages in no order, the free ones on the stack, -1 where a sequence holds no page."""
    order = torch.randperm(_pool(c), generator=_host(seed, 17)).tolist()
    table, at = [], 0
    for n in c["lens"]:
        table.append(order[at:at + _held(c, n)] + [-1] * (c["max_pages"] - _held(c, n)))
        at += _held(c, n)
    return table, order[at:] + [-1] * at


def _rope_inputs(c, seed):
    """Queries and keys as columns of one projection's output (values behind them), and each row's place."""
    g, (h, kv, d) = _gen(seed, 2), (c["heads"], c["kv_heads"], c["d"])
    qkv = _normal(g, (c["rows"], (h + 2 * kv) * d), 1.0, _dtype(c["in"]))
    pos = torch.randint(0, c["most"], (c["rows"],), generator=_host(seed, 3), dtype=torch.int32).to(DEV)
    return qkv[:, :h * d].view(-1, h, d), qkv[:, h * d:(h + kv) * d].view(-1, kv, d), pos


ROPE = {"theta": 10000.0, "factor": 8.0, "original_len": 8192.0, "low_turns": 1.0, "high_turns": 4.0}
AMPLITUDE = {"plain": 1.0, "linear": 1.0, "base": 1.0, "turns": 1.2079}


def _adapter_of_rows(c, seed):
    """Runs of rows of one request, each with an adapter or, one in nine, without."""
    g = _host(seed, 5)
    out = []
    while len(out) < c["rows"]:
        a = int(torch.randint(0, c["slots"], (1,), generator=g)) if c["run"] > 1 else (len(out) * 7 + seed) % c["slots"]
        a = -1 if c["rows"] > 8 and int(torch.randint(0, 9, (1,), generator=g)) == 0 else a
        out += [a] * (1 if c["run"] == 1 else 1 + int(torch.randint(0, 2 * c["run"], (1,), generator=g)))
    return out[:c["rows"]]


def _ranks(c):
    """Adapters of several ranks up to the largest, every second one of the largest."""
    r = c["max_rank"]
    return [r if i % 2 == 0 else max(1, r // 2 if i % 4 == 1 else r - 3) for i in range(c["slots"])]


def _adapter_inputs(c, seed):
    g = _gen(seed, 6)
    x = _normal(g, (c["rows"], c["k"]), 1.0, torch.bfloat16)
    base = _normal(g, (c["splits"], c["rows"], c["n"]), 1.3 / math.sqrt(c["splits"]))
    weights = [(_normal(g, (r, c["k"]), 1 / math.sqrt(c["k"]), torch.bfloat16), _normal(g, (c["n"], r), 0.02, torch.bfloat16), 16.0 / r) for r in _ranks(c)]
    return x, base, weights, _ints(_adapter_of_rows(c, seed))


def _sample_inputs(c, seed):
    """Logits as a head leaves them: most of the vocabulary in a bell, a few tokens far above, some forbidden."""
    g, h, (m, v) = _gen(seed, 8), _host(seed, 9), (c["rows"], c["vocab"])
    held = m + m // 2 + 1 if c["mapped"] else m
    z = torch.empty(held, v, dtype=_dtype(c["dtype"]), device=DEV)
    for at in range(0, held, 256):
        part = _normal(g, (min(256, held - at), v), 2.0)
        some = torch.randint(0, v, (part.shape[0], 12), generator=g, device=DEV)
        part.scatter_add_(1, some, torch.empty(some.shape, device=DEV).uniform_(2.0, 11.0, generator=g))
        part[:, v - max(1, v // 200):] = float("-inf")
        z[at:at + part.shape[0]] = part.to(z.dtype)
    pick = lambda values: torch.tensor(values)[torch.randint(0, len(values), (m,), generator=h)].to(DEV)  # noqa: E731
    k = c["top_k"]
    return {"logits": z, "row_map": torch.randperm(held, generator=h)[:m].int().to(DEV) if c["mapped"] else None,
            "temperature": pick([1.0, 1.0, 0.7, 1.3, 0.0]), "top_k": pick([k, k, max(1, k // 2), 0]).int() if k else None,
            "top_p": pick([0.9, 0.95, 0.8, 1.0]) if c["top_p"] else None, "min_p": pick([0.05, 0.02, 0.0]) if c["min_p"] else None,
            "uniform": torch.rand(m, generator=h).to(DEV)}


def prepare(case, seed):
    c = _opened(case)
    st = {"c": c}
    if own:
        from paper_2602_06412_amd import binding as B
        st["B"] = B
    if c["kind"] == "pages":
        table, free = _page_inputs(c, seed)
        b, p, n, rows = len(c["lens"]), c["max_pages"], _pool(c), c["rows"]
        st["from"] = {"page_table": _ints(table), "seq_len": _ints(c["lens"]), "free_pages": _ints(free), "n_free": _ints([c["spare"]])}
        st["want"] = _ints(c["want"])
        st["cu"] = torch.empty(b + 1, dtype=torch.int32, device=DEV)
        st["pos"], st["len"], st["seq"] = (torch.full((rows,), -1, dtype=torch.int32, device=DEV) for _ in range(3))
        st["slot"] = torch.full((rows,), -1, dtype=torch.int64, device=DEV)
        if own:
            st["pages"], st["to"] = (B.KV8Pages(n, c["page"], b, p, DEV) for _ in range(2))
            for name, t in st["from"].items():
                getattr(st["pages"], name).copy_(t.view_as(getattr(st["pages"], name)))
    elif c["kind"] == "rope":
        st["q"], st["k"], st["pos"] = _rope_inputs(c, seed)
        st["m"] = _ints([c["rows"]])
        if own:
            st["freqs"] = torch.empty(c["rot"] // 2, dtype=torch.float64, device=DEV)
            B.sl_rope_freqs(st["freqs"], **({"theta": ROPE["theta"]} if c["scaling"] == "plain" else dict(ROPE, scaling=c["scaling"])))
            st["q_out"], st["k_out"] = (torch.empty(t.shape, dtype=_dtype(c["out"]), device=DEV) for t in (st["q"], st["k"]))
        else:
            st["freqs"] = _freqs(c)
    elif c["kind"] == "adapters":
        st["x"], st["base"], st["weights"], st["which"] = _adapter_inputs(c, seed)
        st["m"] = _ints([c["rows"]])
        if own:
            st["ad"] = B.Adapters(c["slots"], c["max_rank"], c["n"], c["k"], DEV)
            for slot, (a, b, scale) in enumerate(st["weights"]):
                B.sl_adapters_pack(st["ad"], slot, a, b, scale)
            st["y"] = torch.empty(c["rows"], c["n"], dtype=_dtype(c["out"]), device=DEV)
            st["workspace"] = torch.empty(B.sl_adapters_workspace_bytes(st["ad"], c["rows"]), dtype=torch.uint8, device=DEV)
    else:
        st.update(_sample_inputs(c, seed))
        st["m"] = _ints([c["rows"]])
        if own:
            st["token"], st["kept"] = (torch.empty(c["rows"], dtype=torch.int32, device=DEV) for _ in range(2))
            st["prob"] = torch.empty(c["rows"], device=DEV)
            st["workspace"] = torch.empty(B.sl_sample_filtered_bytes(c["rows"], c["vocab"]), dtype=torch.uint8, device=DEV)
    return st


# ---- one pass ---------------------------------------------------------------------------------------
def _plain_pages(st):
    c, (table, lens, free, n_free) = st["c"], (st["from"][n] for n in ("page_table", "seq_len", "free_pages", "n_free"))
    b, p, page, rows = len(c["lens"]), c["max_pages"], c["page"], c["rows"]
    want = torch.where(st["want"] < 0, lens, st["want"]).long()
    lens, n_free = lens.long(), n_free.long()
    pages = lambda n: (n + page - 1) // page  # noqa: E731
    had = pages(lens)
    released = (had - pages(want)).clamp(min=0)
    need, more = (pages(want) - had).clamp(min=0), (want - lens).clamp(min=0)
    left, room, granted = n_free[0] + released.sum(), torch.tensor(rows, device=DEV), []
    for i in range(b):
        ok = (need[i] <= left) & (more[i] <= room) & (want[i] <= p * page)
        left, room = left - torch.where(ok, need[i], 0), room - torch.where(ok, more[i], 0)
        granted.append(ok)
    granted = torch.stack(granted)
    new = torch.where((want <= lens) | granted, want, lens)
    need, more = torch.where(granted, need, 0), torch.where(granted, more, 0)
    gone, taken = released.cumsum(0) - released, need.cumsum(0) - need
    n_gone, n_taken = released.sum(), need.sum()
    at = torch.arange(p, device=DEV)[None]
    leaves, comes = (at >= pages(new)[:, None]) & (at < had[:, None]), (at >= had[:, None]) & (at < pages(new)[:, None])
    leaving = torch.where(leaves, gone[:, None] + at - pages(new)[:, None], b * p)                  # its number among the released
    pool = torch.full((b * p + 1,), -1, dtype=torch.int32, device=DEV).scatter_(0, leaving.view(-1), table.reshape(-1))
    coming = (taken[:, None] + at - had[:, None]).clamp(0, b * p)
    from_stack = free[(n_free - 1 - (coming - n_gone)).clamp(0, free.numel() - 1)]
    out = torch.where(comes, torch.where(coming < n_gone, pool[coming], from_stack), torch.where(leaves, -1, table))
    i = torch.arange(free.numel(), device=DEV)
    stack = torch.where((i >= n_free) & (i < n_free + n_gone - n_taken), pool[(n_taken + i - n_free).clamp(0, b * p)], free)
    cu = torch.cat([more.new_zeros(1), more.cumsum(0)])
    r = torch.arange(rows, device=DEV)
    seq = (cu[None, 1:] <= r[:, None]).sum(1).clamp(max=b - 1)
    pos = lens[seq] + r - cu[seq]
    there = r < cu[b]
    slot = out[seq, (pos // page).clamp(0, p - 1)].long() * page + pos % page
    keep = lambda x, old: torch.where(there, x, old).to(old.dtype)  # noqa: E731
    return [out, new.int(), stack, (n_free + n_gone - n_taken).int(), cu.int(), keep(pos, st["pos"]), keep(pos + 1, st["len"]), keep(seq, st["seq"]),
            keep(slot, st["slot"])]


def _freqs(c):
    """Radians a slot, one for each pair."""
    rot, r = c["rot"], ROPE
    theta = r["theta"] * (r["factor"] ** (rot / (rot - 2)) if c["scaling"] == "base" else 1.0)
    f = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    if c["scaling"] == "linear":
        f = f / r["factor"]
    if c["scaling"] == "turns":
        part = ((r["original_len"] * f / (2 * math.pi) - r["low_turns"]) / (r["high_turns"] - r["low_turns"])).clamp(0, 1)
        f = f * (part + (1 - part) / r["factor"])
    return f


def _plain_rope(st):
    c = st["c"]
    rot, half = c["rot"], c["rot"] // 2
    angle = st["pos"].double()[:, None] * st["freqs"][None]
    cos, sin = ((f(angle) * AMPLITUDE[c["scaling"]]).float()[:, None] for f in (torch.cos, torch.sin))
    out = []
    for x in (st["q"], st["k"]):
        y = x.float().clone()
        a, b = (x[..., 0:rot:2].float(), x[..., 1:rot:2].float()) if c["interleaved"] else (x[..., :half].float(), x[..., half:rot].float())
        to = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, half), slice(half, rot))
        y[..., to[0]], y[..., to[1]] = a * cos - b * sin, a * sin + b * cos
        out.append(y.to(_dtype(c["out"])))
    return out


def _plain_adapters(st):
    y, x = st["base"].sum(0), st["x"].float()
    for i, (a, b, scale) in enumerate(st["weights"]):
        y = y + torch.where((st["which"] == i)[:, None], scale * ((x @ a.float().T) @ b.float().T), 0.0)
    return y.to(_dtype(st["c"]["out"]))


def _plain_sample(st):
    c = st["c"]
    z = st["logits"] if st["row_map"] is None else st["logits"][st["row_map"].long()]
    z = z.float()
    z = torch.where(torch.isnan(z), float("-inf"), z)
    v, temperature = c["vocab"], st["temperature"]
    most = z.amax(1, keepdim=True)
    greedy = ~(temperature > 0)
    heat = torch.where(greedy, 1.0, temperature).double()[:, None]
    w = torch.where(z == most, UNIT, torch.round(torch.exp((z.double() - most.double()) / heat) * UNIT)).long()
    w = torch.where(z > float("-inf"), w, 0)
    order = torch.sort(z, dim=1, descending=True, stable=True).indices
    ws, count = w.gather(1, order), (z > float("-inf")).sum(1)
    k = count if st["top_k"] is None else torch.where(st["top_k"] > 0, torch.minimum(st["top_k"], count), count)
    k = torch.where(greedy, torch.minimum(count, count.new_ones(1)), k).long()
    place = torch.arange(v, device=DEV)[None]
    ws = torch.where(place < k[:, None], ws, 0)
    if st["top_p"] is not None:
        running = ws.cumsum(1)
        before = running - ws
        short = before.double() < st["top_p"].double()[:, None] * running[:, -1:].double()
        fewest = (short & (place < k[:, None])).sum(1).clamp(min=1)
        k = torch.where(st["top_p"] < 1, torch.minimum(k, fewest), k)
    if st["min_p"] is not None:
        enough = ((ws.double() >= st["min_p"].double()[:, None] * UNIT) & (place < k[:, None])).sum(1).clamp(min=1)
        k = torch.where(st["min_p"] > 0, torch.minimum(k, enough), k)
    kept = torch.zeros_like(w, dtype=torch.bool).scatter_(1, order, place < k[:, None])
    running = torch.where(kept, w, 0).cumsum(1)
    whole = running[:, -1]
    token = (running.double() <= st["uniform"].double()[:, None] * whole[:, None].double()).sum(1).clamp(max=v - 1)
    weight = w.gather(1, token[:, None])[:, 0]
    return [token.int(), (weight.double() / whole.double()).float(), k.int()]


def run(st):
    c = st["c"]
    if not own:
        return {"pages": _plain_pages, "rope": _plain_rope, "adapters": _plain_adapters, "sample": _plain_sample}[c["kind"]](st)
    B = st["B"]
    if c["kind"] == "pages":
        to = st["to"]
        B.sl_kv8_pages_resize(st["pages"], st["want"], st["cu"], st["pos"], c["rows"], to=to, row_len=st["len"], row_seq=st["seq"], row_slot=st["slot"])
        return [to.page_table, to.seq_len, to.free_pages, to.n_free, st["cu"], st["pos"], st["len"], st["seq"], st["slot"]]
    if c["kind"] == "rope":
        B.sl_rope_rows(st["q"], st["q_out"], st["k"], st["k_out"], st["freqs"], st["pos"], st["m"], c["rows"], interleaved=c["interleaved"],
                       amplitude=AMPLITUDE[c["scaling"]])
        return [st["q_out"], st["k_out"]]
    if c["kind"] == "adapters":
        y = {"y_bf16": st["y"]} if c["out"] == "bf16" else {"y_f32": st["y"]}
        B.sl_adapters_forward(st["ad"], st["x"], st["which"], st["m"], c["rows"], st["workspace"], base=st["base"], splits=c["splits"], **y)
        return st["y"]
    B.sl_sample_filtered(st["logits"], st["m"], c["rows"], st["uniform"], st["token"], st["workspace"], temperature=st["temperature"], top_k=st["top_k"],
                         top_p=st["top_p"], min_p=st["min_p"], row_map=st["row_map"], prob=st["prob"], kept=st["kept"])
    return [st["token"], st["prob"], st["kept"]]


# ---- the same in 64 bits ------------------------------------------------------------------------------
def _resized(c, table=None, free=None):
    """The pages of a case, one after another: (table, stack, its height, lengths, rows as (place, sequence, slot))."""
    table = [list(t) for t in table] if table else [[0] * c["max_pages"] for _ in c["lens"]]
    free = list(free) if free else [0] * _pool(c)
    new, queue, rows, height = list(c["lens"]), [], [], c["spare"]
    for b, (n, w) in enumerate(zip(c["lens"], c["want"])):
        if 0 <= w < n:
            for i in range(_held(c, w), _held(c, n)):
                queue.append(table[b][i])
                table[b][i] = -1
            new[b] = w
    left, room = height + len(queue), c["rows"]
    out_of_queue = 0
    for b, (n, w) in enumerate(zip(c["lens"], c["want"])):
        need = _held(c, w) - _held(c, n)
        if w <= n or need > left or w - n > room or w > c["max_pages"] * c["page"]:
            continue
        left, room, new[b] = left - need, room - (w - n), w
        for i in range(_held(c, n), _held(c, w)):
            if out_of_queue < len(queue):
                table[b][i] = queue[out_of_queue]
                out_of_queue += 1
            else:
                height -= 1
                table[b][i] = free[height]
        rows += [(s, b, table[b][s // c["page"]] * c["page"] + s % c["page"]) for s in range(n, w)]
    for page in queue[out_of_queue:]:
        free[height] = page
        height += 1
    return table, free, height, new, rows


def _exact_pages(c, seed):
    table, free, height, new, rows = _resized(c, *_page_inputs(c, seed))
    starts = [0]
    for n, old in zip(new, c["lens"]):
        starts.append(starts[-1] + max(0, n - old))
    pad = [-1] * (c["rows"] - len(rows))
    pos, seq, slot = ([r[i] for r in rows] for i in range(3))
    return [_ints(table), _ints(new), _ints(free), _ints([height]), _ints(starts), _ints(pos + pad), _ints([p + 1 for p in pos] + pad), _ints(seq + pad),
            _ints(slot + pad, torch.int64)]


def _exact_rope(c, seed):
    q, k, pos = _rope_inputs(c, seed)
    per_slot = []                                           # turns of each pair
    for j in range(c["rot"] // 2):
        theta = ROPE["theta"] * ROPE["factor"] ** (c["rot"] / (c["rot"] - 2)) if c["scaling"] == "base" else ROPE["theta"]
        f = math.exp(-2.0 * j / c["rot"] * math.log(theta)) / (2 * math.pi)
        if c["scaling"] == "linear":
            f /= ROPE["factor"]
        if c["scaling"] == "turns":
            over = ROPE["original_len"] * f
            part = min(1.0, max(0.0, (over - ROPE["low_turns"]) / (ROPE["high_turns"] - ROPE["low_turns"])))
            f = part * f + (1 - part) * f / ROPE["factor"]
        per_slot.append(f)
    turns = torch.outer(pos.double(), torch.tensor(per_slot, dtype=torch.float64, device=DEV))
    turns = (turns - turns.round()) * (2 * math.pi)
    turn = torch.polar(torch.full_like(turns, AMPLITUDE[c["scaling"]]), turns)[:, None]
    out = []
    for x in (q.double(), k.double()):
        head, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        pairs = head.unflatten(-1, (-1, 2)) if c["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        out.append(torch.cat([(y if c["interleaved"] else y.transpose(-1, -2)).flatten(-2), rest], -1))
    return out


def _exact_adapters(c, seed):
    x, base, weights, which = _adapter_inputs(c, seed)
    y = base.double().sum(0)
    which = which.tolist()
    for i, (a, b, scale) in enumerate(weights):
        rows = [r for r, w in enumerate(which) if w == i]
        if rows:
            y[rows] += (x[rows].double() @ a.double().t()) @ (b.double().t() * scale)
    return y


def _exact_sample(c, seed):
    s = _sample_inputs(c, seed)
    value = lambda name, r, off: off if s[name] is None else s[name][r].item()  # noqa: E731
    tokens, probs, counts = [], [], []
    for r in range(c["rows"]):
        z = s["logits"][r if s["row_map"] is None else int(s["row_map"][r])].double()
        ids = torch.nonzero(z > float("-inf"))[:, 0]
        z = z[ids]
        heat = value("temperature", r, 1.0)
        falling, where = z.sort(descending=True, stable=True)
        weight = ((falling - falling[0]) / heat).exp().mul(UNIT).round() / UNIT if heat > 0 else (torch.arange(len(z), device=DEV) == 0).double()
        size = 1 if not heat > 0 else len(z)
        k, p, least = int(value("top_k", r, 0)), value("top_p", r, 1.0), value("min_p", r, 0.0)
        if k > 0:
            size = min(size, k)
        if p < 1:
            mass = weight[:size].cumsum(0)
            size = min(size, 1 + int(torch.searchsorted(mass, p * mass[-1])))
        if least > 0:
            size = min(size, max(1, int((weight >= least).sum())))
        chosen, at = where[:size].sort()
        mass = weight[:size][at].cumsum(0)
        i = min(int(torch.searchsorted(mass, value("uniform", r, 0.0) * mass[-1], right=True)), size - 1)
        tokens.append(int(ids[chosen[i]]))
        probs.append(float(weight[at[i]] / mass[-1]))
        counts.append(size)
    return [_ints(tokens), torch.tensor(probs, dtype=torch.float64, device=DEV), _ints(counts)]


def exact(case, seed):
    c = _opened(case)
    return {"pages": _exact_pages, "rope": _exact_rope, "adapters": _exact_adapters, "sample": _exact_sample}[c["kind"]](c, seed)
