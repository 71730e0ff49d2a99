"""Plain definitions of the serving-step operators (not collected by pytest): what sl_kv8_pages_*, sl_rope_*, sl_adapters_* and
sl_sample_filtered compute, written from their definitions with NumPy in 64 bits and whole numbers."""
import math

import numpy as np

UNIT = 2.0 ** 44


# ---- pages ---------------------------------------------------------------------------------------
def pages_resize(table, lens, stack, n_free, want, page, n_pages, m_upper):
    """Lists in, lists out: (table, lens, stack, n_free, cu_rows, rows as (pos, seq, slot))."""
    table, stack, max_pages = [list(t) for t in table], list(stack), len(table[0])
    held = lambda n: -(-n // page)  # noqa: E731
    lens = [min(max(n, 0), max_pages * page) for n in lens]
    n_free = min(max(n_free, 0), n_pages)
    want = [n if w < 0 else w for n, w in zip(lens, want)]
    new, queue = list(lens), []
    for b, (n, w) in enumerate(zip(lens, want)):
        for i in range(held(w), held(n)):
            queue.append(table[b][i])
            table[b][i] = -1
        new[b] = min(n, w)
    left, room, rows, cu = n_free + len(queue), m_upper, [], [0]
    for b, (n, w) in enumerate(zip(lens, want)):
        need = held(w) - held(n)
        if w > n and w <= max_pages * page and need <= left and w - n <= room:
            left, room, new[b] = left - need, room - (w - n), w
            for i in range(held(n), held(w)):
                if queue:
                    table[b][i] = queue.pop(0)
                else:
                    n_free -= 1
                    table[b][i] = stack[n_free]
            for s in range(n, w):
                p = table[b][s // page]
                rows.append((s, b, p * page + s % page if 0 <= p < n_pages else -1))
        cu.append(len(rows))
    for p in queue:
        if n_free < n_pages:
            stack[n_free] = p
            n_free += 1
    return table, new, stack, n_free, cu, rows


# ---- rotary positions ------------------------------------------------------------------------------
def rope_freqs(rot, theta, scaling="plain", factor=1.0, original_len=0.0, low=0.0, high=0.0):
    """Turns a slot."""
    if scaling == "base":
        theta = theta * factor ** (rot / (rot - 2))
    f = np.array([theta ** (-2.0 * j / rot) / (2 * math.pi) for j in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "turns":
        g = np.clip((original_len * f - low) / (high - low), 0, 1)
        f = f * g + (1 - g) * f / factor
    return f


def rope_rows(x, pos, freqs, interleaved, amplitude):
    """x [rows, heads, d] float64 -> (y, |a| + |b| of each number's pair; 0 where nothing turns)."""
    rot = 2 * len(freqs)
    # whole turns fall away in extended precision: a position times a frequency has more bits than a float64
    turns = np.asarray(pos, np.longdouble)[:, None] * np.asarray(freqs, np.longdouble)[None]
    t = ((turns - np.rint(turns)) * (2 * np.pi)).astype(np.float64)[:, None]
    c, s = amplitude * np.cos(t), amplitude * np.sin(t)
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    y, mass = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    mass[..., a] = mass[..., b] = abs(amplitude) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, mass


def rope_bound(y, mass, eps_out):
    """|error|: sine and cosine (times the amplitude) are off by half a step of fp32 and what Taylor's sums and the angle leave (2^-33), a
    product and a sum round once each; then the result's own rounding, half a step."""
    return mass * (2.0 ** -24 + 2.0 ** -33 + 2 * 2.0 ** -24) + (np.abs(y) + mass * 2.0 ** -22) * eps_out / 2 + 1e-37


# ---- adapters --------------------------------------------------------------------------------------
def adapters(x, base, which, weights):
    """x [m, k], base [s, m, n] or None, weights: {slot: (a [r, k], b [n, r], scale)} (float64) -> (y, error bound without the result's rounding)."""
    m, n = x.shape[0], base.shape[2] if base is not None else next(iter(weights.values()))[1].shape[0]
    y, size = np.zeros((m, n)), np.zeros((m, n))
    if base is not None:
        y, size = base.sum(0), (base.shape[0] + 1) * 2.0 ** -24 * np.abs(base).sum(0)
    for r, w in enumerate(which):
        if w in weights:
            a, b, scale = weights[w]
            h = a @ x[r]
            h_size = np.abs(a) @ np.abs(x[r])
            y[r] += scale * (b @ h)
            # sums of k terms in any order, then of three parts of each of rank terms; scale, the parts' last rounding, the final sum
            size[r] += abs(scale) * (np.abs(b) @ h_size) * (x.shape[1] + 3 * a.shape[0] + 16) * 2.0 ** -24
    return y, size + 2.0 ** -24 * np.abs(y)


# ---- draws -----------------------------------------------------------------------------------------
def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row (float64) -> (token, prob, kept)."""
    ids = np.nonzero(z > -np.inf)[0]
    if not len(ids):
        return 0, 0.0, 0
    order = ids[np.lexsort((ids, -z[ids]))]
    most = z[order[0]]
    if not temperature > 0:
        return int(order[0]), 1.0, 1
    with np.errstate(all="ignore"):
        w = np.where(z[order] == most, UNIT, np.rint(np.exp((z[order] - most) / temperature) * UNIT) if np.isfinite(most) else 0.0)
    w = w.astype(np.int64)                                       # (sums stay below 2^63)
    size = len(w) if top_k <= 0 else min(top_k, len(w))
    if top_p < 1:
        run = w[:size].cumsum()
        size = max(1, min(size, 1 + int((run.astype(np.float64) < float(top_p) * float(run[-1])).sum())))
    if min_p > 0:
        size = max(1, min(size, int((w.astype(np.float64) >= float(min_p) * UNIT).sum())))
    by_id = np.argsort(order[:size])
    chosen, w = order[:size][by_id], w[:size][by_id]
    run = w.cumsum()
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    i = int((run.astype(np.float64) <= u * float(run[-1])).sum())
    return int(chosen[i]), float(w[i]) / float(run[-1]), size
