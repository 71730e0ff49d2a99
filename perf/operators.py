"""The low-bit operators of few-row decoding, over the sizes a decoding program meets, for measuring them.

Late in a run few rows per sequence are still active, and a block's time goes into streaming its weights and its K/V
cache.  Three operators make both streams shorter:

  linear     y = x W^T with 4-bit weights and one scale (and zero point) per group of inputs (sl_linear_q4_forward)
  cache      rows of K and V quantised to 8 bits as they are written into a paged cache, and read back (sl_kv8_write,
             sl_kv8_read)
  attention  the rows' attention over the slots of their sequence in that cache (sl_kv8_attention)

`own` chooses between the plain formulas below and the library's kernels.  Definitions:

  weights    W[j, i] = scales[j, i / group] * (code[j, i] - zeros[j, i / group]), codes 0..15, two to a byte, the lower
             half first; without zero points they are 8
  cache      per row and head: scale = max|x| / 127 in fp32 (0 for a zero vector, NaN unless all are finite), code =
             rint(x / scale), the quotient in fp32; the value is code * scale
  attention  softmax over the first min(seq_len, row_len) slots, zeros where there are none
"""
import math

import torch

own = False
DEV = "cuda:0"
LLADA_D, LLADA_HEADS, LLADA_HEAD, LLADA_FF = 4096, 32, 128, 12288          # the LLaDA-8B-shaped block
TINY_D, TINY_HEADS, TINY_HEAD, TINY_FF = 256, 4, 64, 688                   # the tiny fp32 model


# ---- the cases ------------------------------------------------------------------------------------
def listed():
    return [
        # the tiny model's gate projection for one row: launch and latency; 688 columns are no multiple of a tile
        {"name": "linear_tiny_m1", "kind": "linear", "rows": 1, "n": TINY_FF, "k": TINY_D, "group": 32, "zeros": False, "out": "fp32"},
        # one row left in one sequence: the Out projection, the smallest of a block
        {"name": "linear_out_m1", "kind": "linear", "rows": 1, "n": LLADA_D, "k": LLADA_D, "group": 128, "zeros": False, "out": "bf16"},
        # the last step of a short sequence: the fused Q|K|V projection, with zero points
        {"name": "linear_qkv_m16", "kind": "linear", "rows": 16, "n": 3 * LLADA_D, "k": LLADA_D, "group": 128, "zeros": True, "out": "bf16"},
        # the last step of a long sequence, an odd row count: the down projection, fine groups
        {"name": "linear_down_m61", "kind": "linear", "rows": 61, "n": LLADA_D, "k": LLADA_FF, "group": 64, "zeros": False, "out": "bf16"},
        # the later half of a short sequence's schedule: the gate|up projection, the largest product
        {"name": "linear_gate_up_m224", "kind": "linear", "rows": 224, "n": 2 * LLADA_FF, "k": LLADA_D, "group": 128, "zeros": True, "out": "bf16"},
        # three rows of the tiny model: latency of the write and of the reading
        {"name": "cache_tiny_m3", "kind": "cache", "dtype": "fp32", "heads": TINY_HEADS, "d": TINY_HEAD, "page": 16, "lens": "128",
         "rows": "3"},
        # a late step of a batch of eight: scattered active rows, ragged counts
        {"name": "cache_8x1024_m137", "kind": "cache", "dtype": "bf16", "heads": LLADA_HEADS, "d": LLADA_HEAD, "page": 64, "lens": "1024 1024 1024 1024 1024 1024 1024 1024",
         "rows": "3 8 12 16 19 22 26 31"},
        # the first step of a batch of eight ragged sequences: every slot is written
        {"name": "cache_8_prompts", "kind": "cache", "dtype": "bf16", "heads": LLADA_HEADS, "d": LLADA_HEAD, "page": 64,
         "lens": "1024 77 640 1024 333 911 500 1024", "rows": "1024 77 640 1024 333 911 500 1024"},
        # the tiny model, three rows of one sequence: latency
        {"name": "attention_tiny_m3", "kind": "attention", "dtype": "fp32", "heads": TINY_HEADS, "kv_heads": TINY_HEADS, "d": TINY_HEAD,
         "page": 16, "lens": "128", "rows": "3", "row_len": False},
        # the last step of a long sequence: 64 rows over all its slots
        {"name": "attention_2048_m64", "kind": "attention", "dtype": "bf16", "heads": LLADA_HEADS, "kv_heads": LLADA_HEADS, "d": LLADA_HEAD,
         "page": 64, "lens": "2048", "rows": "64", "row_len": False},
        # one row in each of eight ragged sequences, every head with keys of its own
        {"name": "attention_8_ragged_m1", "kind": "attention", "dtype": "bf16", "heads": LLADA_HEADS, "kv_heads": LLADA_HEADS,
         "d": LLADA_HEAD, "page": 64, "lens": "4096 1025 7000 300 2048 5555 63 8192", "rows": "1 1 1 1 1 1 1 1", "row_len": False},
        # long sequences, heads that share keys, one to four rows each, a row sees the slots up to its own: the largest cache
        {"name": "attention_16_long_shared", "kind": "attention", "dtype": "bf16", "heads": 32, "kv_heads": 8, "d": 128, "page": 128,
         "lens": "32768 20011 31999 8192 27000 16384 32768 24681 30000 12345 32001 29999 4097 32768 21000 26000",
         "rows": "1 2 4 1 3 1 2 1 4 1 1 2 1 4 1 3", "row_len": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _opened(c):
    """The case with its lists (a number a sequence, as text) as lists."""
    return {n: [int(x) for x in v.split()] if n in ("lens", "rows") and isinstance(v, str) else v for n, v in c.items()}


def _cost(c):
    """A rough time, to keep drawn cases below the largest listed one of their kind."""
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 4e14


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    kind = rng.choice(["linear", "linear", "cache", "attention", "attention"])
    while True:
        if kind == "linear":
            n = rng.choice([_log_int(rng, 64, 2 * LLADA_FF), 32 * _log_int(rng, 2, 768), rng.choice([TINY_FF, LLADA_D, LLADA_FF, 2 * LLADA_FF])])
            k = rng.choice([8 * _log_int(rng, 8, LLADA_FF // 8), 128 * _log_int(rng, 1, LLADA_FF // 128), rng.choice([TINY_D, TINY_FF, LLADA_D, LLADA_FF])])
            c = {"kind": kind, "rows": _log_int(rng, 1, 256), "n": n, "k": k, "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.5,
                 "out": rng.choice(["bf16", "bf16", "fp32"])}
        elif kind == "cache":
            lens = [_log_int(rng, 1, 2048) for _ in range(rng.randint(1, 12))]
            c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "fp32"]), "heads": rng.choice([1, 2, 4, 8, 16, 32]),
                 "d": rng.choice([32, 64, 128, 128, 256]), "page": rng.choice([16, 32, 64, 128, 256]), "lens": lens,
                 "rows": [n if rng.random() < 0.4 else _log_int(rng, 1, n) for n in lens]}
        else:
            kv = rng.choice([1, 2, 4, 8, 8, 32])
            share = rng.choice([1, 2, 4, 8]) if kv < 32 else 1
            lens = [_log_int(rng, 1, 32768) for _ in range(rng.randint(1, 16))]
            c = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "heads": kv * share, "kv_heads": kv,
                 "d": rng.choice([32, 64, 128, 128, 128, 256]), "page": rng.choice([16, 32, 64, 128, 256]), "lens": lens,
                 "rows": [min(n, rng.choice([1, 1, _log_int(rng, 1, 64)])) for n in lens], "row_len": rng.random() < 0.5}
        if _cost(c) <= most[kind]:
            return {n: " ".join(map(str, v)) if isinstance(v, list) else v for n, v in c.items()}


def work(c):
    """Each input once and each output once; a sequence's cache as far as its rows see it."""
    c = _opened(c)
    if c["kind"] == "linear":
        groups = c["n"] * -(-c["k"] // c["group"])
        return {"bytes": c["n"] * c["k"] / 2 + groups * (3 if c["zeros"] else 2) + c["rows"] * (2.0 * c["k"] + c["n"] * (2 if c["out"] == "bf16" else 4)),
                "flops": 2.0 * c["rows"] * c["n"] * c["k"]}
    ts = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "cache":
        vectors = 2.0 * sum(c["rows"]) * c["heads"]
        return {"bytes": vectors * 2 * (c["d"] * (ts + 1) + 4), "flops": vectors * c["d"] * 4}
    pairs = 0.0
    for n, m in zip(c["lens"], c["rows"]):
        pairs += sum(_seen(n, m)) if c["row_len"] else n * m
    return {"bytes": 2.0 * sum(c["lens"]) * c["kv_heads"] * (c["d"] + 4) + 2.0 * sum(c["rows"]) * c["heads"] * c["d"] * ts,
            "flops": 4.0 * pairs * c["heads"] * c["d"]}


def _seen(n, m):
    """How many slots each of the last m rows of a sequence of n sees, its own among them."""
    return [n - m + 1 + i for i in range(m)]


# ---- inputs, from the seed alone --------------------------------------------------------------------
def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + what) % (1 << 62))


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, std, generator=gen).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _linear_inputs(c, seed):
    """Rows as a norm leaves them, weights N(0, 0.02^2) rounded to the nearest code of their group."""
    g = _gen(seed, 1)
    n, k, gr = c["n"], c["k"], c["group"]
    x = _normal(g, (c["rows"], k), 1.0, torch.bfloat16)
    groups = -(-k // gr)
    w = torch.zeros(n, groups * gr, device=DEV)
    w[:, :k] = _normal(g, (n, k), 0.02)
    w = w.view(n, groups, gr)
    if c["zeros"]:
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        scales = ((hi - lo) / 15).bfloat16()
        zeros = torch.round(-lo / scales.float()).clamp(0, 15)
    else:
        scales = (w.abs().amax(2) / 7).bfloat16()
        zeros = torch.full_like(scales, 8, dtype=torch.float32)
    codes = (torch.round(w / scales.float()[:, :, None]) + zeros[:, :, None]).clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
    codes = (codes[:, 0::2] | (codes[:, 1::2] << 4)).contiguous()
    return x, codes, scales.contiguous(), zeros.to(torch.uint8).contiguous() if c["zeros"] else None


def _pages(c, seed):
    """A page table [batch, most pages of a sequence]: pages in no order, -1 where a sequence has no more."""
    need = [-(-n // c["page"]) for n in c["lens"]]
    order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(int(seed) + 17)).tolist()
    rows, at = [], 0
    for n in need:
        rows.append(order[at:at + n] + [-1] * (max(need) - n))
        at += n
    return _ints(rows), sum(need)


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return _ints(out)


def _vectors(g, rows, heads, d, dtype):
    """Keys (one dimension in sixteen large, as keys have them) and values, as columns of one projection's output."""
    qkv = _normal(g, (rows, 2 * heads * d))
    qkv[:, :heads * d:16] *= 4.0
    qkv = qkv.to(dtype)
    return qkv[:, :heads * d].view(rows, heads, d), qkv[:, heads * d:].view(rows, heads, d)


def _positions(c, seed):
    """Which slots the rows of each sequence are: some of them, ascending."""
    g = torch.Generator().manual_seed(int(seed) + 29)
    return [torch.randperm(n, generator=g)[:m].sort().values.tolist() for n, m in zip(c["lens"], c["rows"])]


def _cache_inputs(c, seed):
    rows = sum(c["rows"])
    k, v = _vectors(_gen(seed, 2), rows, c["heads"], c["d"], _dtype(c["dtype"]))
    pos = _positions(c, seed)
    return k, v, _ints([p for ps in pos for p in ps]), _starts(c["rows"]), _ints([b for b, ps in enumerate(pos) for _ in ps])


def _sequence(c, seed, b):
    """The keys and values of every slot of sequence b."""
    return _vectors(_gen(seed, 100 + b), c["lens"][b], c["kv_heads"], c["d"], _dtype(c["dtype"]))


def _queries(c, seed):
    # (a spread of scores as trained heads have it: some slots stand out)
    return _normal(_gen(seed, 3), (sum(c["rows"]), c["heads"], c["d"]), 1.0, _dtype(c["dtype"]))


def _row_lens(c):
    return [s for n, m in zip(c["lens"], c["rows"]) for s in (_seen(n, m) if c["row_len"] else [n] * m)]


def prepare(case, seed):
    c = _opened(case)
    st = {"c": c}
    if own:
        from paper_2602_06412_amd import binding as B
        st["B"] = B
    if c["kind"] == "linear":
        st["x"], st["codes"], st["scales"], st["zeros"] = _linear_inputs(c, seed)
        st["m"] = _ints([c["rows"]])
        if own:
            st["packed"] = torch.empty(B.sl_linear_q4_bytes(c["n"], c["k"], c["group"]), dtype=torch.uint8, device=DEV)
            B.sl_linear_q4_pack(st["codes"], st["scales"], st["zeros"], c["n"], c["k"], c["group"], st["packed"])
            st["y"] = torch.empty(c["rows"], c["n"], dtype=_dtype(c["out"]), device=DEV)
        return st
    table, n_pages = _pages(c, seed)
    st["table"] = table
    heads = c["heads"] if c["kind"] == "cache" else c["kv_heads"]
    if own:
        st["kv"] = B.KV8(n_pages, c["page"], heads, c["d"], table)
    else:
        slots = n_pages * c["page"]
        st["codes"] = torch.zeros(2, slots, heads, c["d"], dtype=torch.int8, device=DEV)
        st["scales"] = torch.zeros(2, slots, heads, dtype=torch.float32, device=DEV)
    if c["kind"] == "cache":
        st["k"], st["v"], st["pos"], st["cu"], st["seq"] = _cache_inputs(c, seed)
        if own:
            st["k_out"], st["v_out"] = (torch.empty(sum(c["rows"]), heads, c["d"], dtype=_dtype(c["dtype"]), device=DEV) for _ in range(2))
        return st
    for b, n in enumerate(c["lens"]):
        k, v = _sequence(c, seed, b)
        pos = torch.arange(n, dtype=torch.int32, device=DEV)
        if own:
            B.sl_kv8_write(st["kv"].sequence(b), k, v, pos, _ints([0, n]), n)
        else:
            _write(st, k, v, torch.full_like(pos, b), pos)
    st["q"], st["cu"], st["len"] = _queries(c, seed), _starts(c["rows"]), _ints(c["lens"])
    st["row_len"] = _ints(_row_lens(c)) if c["row_len"] else None
    if own:
        st["out"] = torch.empty_like(st["q"])
        st["workspace"] = torch.empty(B.sl_kv8_attention_bytes(st["kv"], c["heads"], sum(c["rows"]), max(c["lens"])), dtype=torch.uint8, device=DEV)
    return st


# ---- one pass ---------------------------------------------------------------------------------------
def _slots(st, seq, pos):
    page = st["c"]["page"]
    return st["table"][seq.long(), (pos // page).long()].long() * page + (pos % page).long()


def _write(st, k, v, seq, pos):
    at = _slots(st, seq, pos)
    for i, x in enumerate((k, v)):
        x = x.float()
        most = x.abs().amax(-1)
        scale = torch.where(torch.isfinite(most), most / torch.tensor(127.0, device=DEV), float("nan"))
        code = torch.round(x / scale[..., None])
        st["codes"][i][at] = torch.where(scale[..., None] > 0, code, 0.0).to(torch.int8)
        st["scales"][i][at] = scale


def _values(st, i, at):
    return st["codes"][i][at].float() * st["scales"][i][at][..., None]


def _plain_linear(st):
    c = st["c"]
    n, k, gr = c["n"], c["k"], c["group"]
    codes = torch.stack([st["codes"] & 15, st["codes"] >> 4], -1).view(n, k).float()
    spread = lambda t: t.float().repeat_interleave(gr, 1)[:, :k]  # noqa: E731
    w = (codes - (spread(st["zeros"]) if c["zeros"] else 8.0)) * spread(st["scales"])
    return (st["x"].float() @ w.T).to(_dtype(c["out"]))


def _plain_attention(st):
    c = st["c"]
    share, d = c["heads"] // c["kv_heads"], c["d"]
    out = torch.zeros_like(st["q"])
    at = 0
    for b, (n, m) in enumerate(zip(c["lens"], c["rows"])):
        pos = torch.arange(n, device=DEV)
        slots = _slots(st, torch.full_like(pos, b), pos)
        k, v = (_values(st, i, slots).transpose(0, 1).contiguous() for i in (0, 1))             # [kv_heads, n, d]
        q = st["q"][at:at + m].float().view(m, c["kv_heads"], share, d).permute(1, 0, 2, 3).reshape(c["kv_heads"], m * share, d)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        if c["row_len"]:
            hidden = pos[None] >= st["row_len"][at:at + m, None]
            s = s.masked_fill(hidden.repeat_interleave(share, 0)[None], float("-inf"))
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(p / p.sum(-1, keepdim=True), v)
        out[at:at + m] = o.view(c["kv_heads"], m, share, d).permute(1, 0, 2, 3).reshape(m, c["heads"], d).to(out.dtype)
        at += m
    return out


def run(st):
    c = st["c"]
    rows = sum(c["rows"]) if c["kind"] != "linear" else c["rows"]
    if not own:
        if c["kind"] == "linear":
            return _plain_linear(st)
        if c["kind"] == "attention":
            return _plain_attention(st)
        _write(st, st["k"], st["v"], st["seq"], st["pos"])
        at = _slots(st, st["seq"], st["pos"])
        return [_values(st, i, at).to(_dtype(c["dtype"])) for i in (0, 1)]
    B = st["B"]
    if c["kind"] == "linear":
        y = {"y_bf16": st["y"]} if c["out"] == "bf16" else {"y_f32": st["y"]}
        B.sl_linear_q4_forward(st["x"], st["packed"], st["m"], rows, c["n"], c["k"], c["group"], **y)
        return st["y"]
    if c["kind"] == "attention":
        B.sl_kv8_attention(st["kv"], st["q"], st["cu"], st["len"], rows, max(c["lens"]), 1.0 / math.sqrt(c["d"]), st["out"],
                           st["workspace"], row_len=st["row_len"])
        return st["out"]
    B.sl_kv8_write(st["kv"], st["k"], st["v"], st["pos"], st["cu"], rows)
    B.sl_kv8_read(st["kv"], st["k_out"], st["v_out"], st["pos"], st["cu"], rows)
    return [st["k_out"], st["v_out"]]


# ---- the same in 64 bits ------------------------------------------------------------------------------
def _cached64(x):
    """What the cache keeps of x [.., d]; its two quotients are rounded to fp32 by definition, the rest is exact."""
    x = x.double()
    peak = x.abs().max(-1, keepdim=True).values
    step = (peak / 127.0).float().double()
    code = (x / torch.where(step > 0, step, torch.ones_like(step))).float().double().round()
    return code * step


def exact(case, seed):
    c = _opened(case)
    if c["kind"] == "linear":
        x, codes, scales, zeros = _linear_inputs(c, seed)
        out = torch.empty(c["rows"], c["n"], dtype=torch.float64, device=DEV)
        group = torch.arange(c["k"], device=DEV) // c["group"]
        odd = (torch.arange(c["k"], device=DEV) % 2) * 4
        for j in range(0, c["n"], 2048):
            code = (codes[j:j + 2048].repeat_interleave(2, 1) >> odd) & 15
            zero = zeros[j:j + 2048][:, group].double() if zeros is not None else 8.0
            out[:, j:j + 2048] = x.double() @ ((code.double() - zero) * scales[j:j + 2048][:, group].double()).T
        return out
    if c["kind"] == "cache":
        k, v = _cache_inputs(c, seed)[:2]
        return [_cached64(k), _cached64(v)]
    q = _queries(c, seed).double()
    out = torch.zeros_like(q)
    seen, at = _row_lens(c), 0
    for b, m in enumerate(c["rows"]):
        k, v = (_cached64(t) for t in _sequence(c, seed, b))
        for r in range(at, at + m):
            for h in range(c["kv_heads"]):
                share = slice(h * (c["heads"] // c["kv_heads"]), (h + 1) * (c["heads"] // c["kv_heads"]))
                w = torch.softmax((q[r, share] @ k[:seen[r], h].T) / math.sqrt(c["d"]), -1)
                out[r, share] = w @ v[:seen[r], h]
        at += m
    return out
