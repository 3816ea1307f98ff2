"""Oracle (test infrastructure): the operators on packed tokens written out as their definitions, in fp64 numpy.

Attention is given for one query head at a time over the keys that each query may see; bounds() says how far a kernel that
rounds its operands to bf16 and sums in fp32 may be off."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def build_slots(ctx, new, table, free, free_at, T, page):
    """(table, cu, lens, positions, slots, free_next), request by request."""
    table, R, width = table.copy(), len(ctx), table.shape[1]
    positions, slots, cu, lens = np.zeros(T, np.int64), np.full(T, -1, np.int64), [0], []
    at = free_at
    for r in range(R):
        c, a = max(0, int(ctx[r])), max(0, int(new[r]))
        for p in range(min(-(-c // page), width), min(-(-(c + a) // page), width)):
            table[r, p] = free[at] if 0 <= at < len(free) else -1
            at += 1
        for i in range(a):
            t, pos = cu[-1] + i, c + i
            if t < T:
                positions[t] = pos
                if pos // page < width and table[r, pos // page] >= 0:
                    slots[t] = table[r, pos // page] * page + pos % page
        cu.append(cu[-1] + a)
        lens.append(c + a)
    return table, np.array(cu), np.array(lens), positions, slots, at


def rope(x, positions, freqs, interleaved, mscale=1.0, inverse=False):
    """x [T, H, d]; freqs [rot/2]."""
    x, y, rot = np.asarray(x, np.float64), np.array(x, np.float64), 2 * len(freqs)
    a = positions.astype(np.float64)[:, None] * freqs.astype(np.float64) * (-1 if inverse else 1)
    one = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    two = one + (1 if interleaved else rot // 2)
    c, s = mscale * np.cos(a)[:, None], mscale * np.sin(a)[:, None]
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    return y


def attention(q, k, v, seen, scale):
    """q [n, d], k, v [m, d], seen [n, m]: (O, lse, P); a query that sees nothing gets 0 and -inf."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    any_key = seen.any(1)
    top = np.where(any_key, s.max(1, initial=-np.inf), 0.0)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        p = np.exp(s - top[:, None])
        total = p.sum(1)
        p = np.where(any_key[:, None], p / total[:, None], 0.0)
        lse = np.where(any_key, top + np.log(total), -np.inf)
    return p @ np.where(seen.any(0)[:, None], v, 0.0), lse, p


def attention_bwd(q, k, v, d_o, p, scale, delta):
    """(dQ, dK, dV) from P; delta = <dO, O>."""
    ds = p * (d_o @ v.T - delta[:, None])
    return scale * (ds @ k), scale * (ds.T @ q), p.T @ d_o


# Half a step of bf16 and of fp32, relative to the value.
B, F = 2.0 ** -8, 2.0 ** -24
# What falls below the normal range of fp32 is lost: less than 2^-126 of a probability, in each of at most 2^12 terms, times other factors (dP, a query's
# or key's element, the scale) that stay below 2^24 in all.
U = 2.0 ** -90


def bounds(q, k, v, seen, scale, p, o, lse, d_o=None, delta=None, grads=None):
    """How far O, lse (and dQ, dK, dV) may be off: every product of two bf16 numbers is exact in fp32, a sum of d (of n) terms in any order is off
    by at most d (n) half steps of the sum of their magnitudes, an exponential or logarithm by a few steps; P and dS are rounded to bf16
    once each (dS from a rounded P), the results once."""
    d, n = q.shape[1], max(1, int(seen.sum(1).max(initial=0)))
    mag = np.where(seen, scale * (np.abs(q) @ np.abs(k).T), 0.0)
    e_s = (d + 8) * F * mag + 32 * F * (1 + mag)                      # of a score, and of its exponent in units of log2
    e_row = e_s.max(1, initial=0.0)
    vis = np.where(seen.any(0)[:, None], np.abs(v), 0.0)
    a = p @ vis
    e_p = 2 * e_row + (n + 16) * F                                     # of P, relative: its own exponent and the sum's
    e_lse = e_row + (n + 16) * F + 4 * F * np.abs(np.where(np.isfinite(lse), lse, 0.0))
    e_o = U + B * np.abs(o) + (B * (1 + B) + e_p + n * F)[:, None] * a
    if d_o is None:
        return e_o, e_lse
    dq, dk, dv = grads
    dp, dp_mag = np.abs(d_o @ v.T - delta[:, None]), np.abs(d_o) @ np.abs(v).T + (np.abs(d_o) * np.abs(o)).sum(1)[:, None]
    ds = p * dp
    e_p = (e_row + e_lse + 32 * F)[:, None]                            # P from the stored lse, relative
    e_ds = (2 * B + B * B + e_p) * ds + p * (d + 8) * F * dp_mag
    e_dq = U + B * np.abs(dq) + scale * (e_ds @ np.abs(k) + n * F * (ds @ np.abs(k)))
    rows = p.shape[0]
    e_dk = U + B * np.abs(dk) + scale * (e_ds.T @ np.abs(q) + rows * F * (ds.T @ np.abs(q)))
    e_dv = U + B * np.abs(dv) + ((B + e_p) * p).T @ np.abs(d_o) + rows * F * (p.T @ np.abs(d_o))
    return e_o, e_lse, e_dq, e_dk, e_dv


def key_weights(q, k, seen, scale, lse):
    """q [n, d], k [m, d], seen [n, m], lse [n]: (what each key gets, how far a kernel may be off that sums n products in fp32): the probabilities from the given lse."""
    n, d = q.shape
    with np.errstate(invalid="ignore"):
        p = np.where(seen & np.isfinite(lse)[:, None], np.exp(np.where(seen, scale * (q @ k.T) - np.where(np.isfinite(lse), lse, 0.0)[:, None], -np.inf)), 0.0)
    mag = np.where(seen, scale * (np.abs(q) @ np.abs(k).T), 0.0)
    e = (d + 8) * F * mag + 32 * F * (1 + mag + np.abs(np.where(np.isfinite(lse), lse, 0.0))[:, None])   # of an exponent: the score, both in units of log2, their difference
    return p.sum(0), ((2 * e + (n + 16) * F) * p).sum(0) + n * U


def kv4_encode(x):
    """x [..., 32 n] finite: (codes, scale bytes) of groups of 32, by looking at every exponent and every code."""
    x = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, 32))
    exps = np.arange(-120, 126)
    fits = np.abs(x).max(-1)[..., None] <= 7 * 2.0 ** exps
    e = np.where(fits.any(-1), exps[fits.argmax(-1)], 125)
    y = np.abs(x) / (2.0 ** e)[..., None]
    dist = np.abs(y[..., None] - GRID)
    tie_even = np.where(dist == dist.min(-1, keepdims=True), np.arange(8) % 2, 2).argmin(-1)
    return (tie_even + 8 * np.signbit(x)).astype(np.uint8).reshape(x.shape[:-2] + (-1,)), (e + 127).astype(np.uint8)


def kv4_decode(codes, scales):
    """codes [..., 32 n] (one a byte), scale bytes [..., n]."""
    x = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return x * np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, -1)


def unpack_nibbles(b):
    """[..., m] bytes: [..., 2 m] codes."""
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (-1,))


def evict(n, budget, recent, first, w):
    """Which key goes to which position, by pairs (from, to), in one head of a request of n keys with weights w (fp32; -inf for a NaN's place: use None below any number for a key without a page):
    by sorting.  And how many stay."""
    f = max(0, first)
    b = max(budget, f + recent)
    if n <= b:
        return [], n
    size = lambda j: (2, float(w[j])) if w[j] is not None and not np.isnan(w[j]) else ((1, 0.0) if w[j] is not None else (0, 0.0))  # noqa: E731
    between = sorted(range(f, n - recent), key=lambda j: tuple(-x for x in size(j)) + (j,))
    kept, edge = set(between[:b - f - recent]), b - recent
    free = [j for j in range(f, edge) if j not in kept]
    return list(zip(sorted(j for j in kept if j >= edge), free)) + [(n - recent + i, edge + i) for i in range(recent)], b
