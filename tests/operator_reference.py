"""The operators on callers' tensors in 64 bits, from their definitions (numpy; no code of the library)."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}           # half a step, relative


def quantise(x):
    """x [..., 32 n] float64 -> magnitude codes with sign (uint8), scale bytes [..., n]"""
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    a = np.abs(g).max(-1)
    m, e = np.frexp(np.where(a > 0, a, 1.0))
    e = np.where(2 * m <= 1.75, e - 3, e - 2)
    e = np.clip(np.where(a > 0, e, -100), -100, 125)
    y = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    code = np.zeros(y.shape, np.uint8)
    d = np.abs(y[..., None] - LEVELS)
    best = d.min(-1, keepdims=True)
    near = d == best                                         # one code, or two neighbours: the even one
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1)).astype(np.uint8)
    code = code | (np.signbit(g) * 8).astype(np.uint8)
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def values(code, scale):
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return (v.reshape(v.shape[:-1] + (v.shape[-1] // 32, 32)) * s[..., None]).reshape(v.shape)


def chunk_bytes(hd, block):
    return block * (hd + hd // 16)


def split_pool(pool, heads, hd, block):
    """pool bytes -> key codes, value codes [blocks][heads][block][hd], key scales, value scales [..][block][hd / 32] (views of copies)"""
    p = pool.reshape(-1, heads, chunk_bytes(hd, block))
    cut = np.cumsum([0, block * hd // 2, block * hd // 2, block * hd // 32, block * hd // 32])
    k, v, ks, vs = (p[:, :, a:b].reshape(p.shape[0], heads, block, -1) for a, b in zip(cut, cut[1:]))
    wide = lambda c: np.stack((c & 15, c >> 4), -1).reshape(c.shape[:-1] + (2 * c.shape[-1],))
    return wide(k), wide(v), ks, vs


def join_pool(k, v, ks, vs):
    narrow = lambda c: (c[..., ::2] | c[..., 1::2] << 4)
    flat = lambda x: x.reshape(x.shape[0], x.shape[1], -1)
    return np.ascontiguousarray(np.concatenate([flat(narrow(k)), flat(narrow(v)), flat(ks), flat(vs)], -1)).reshape(-1)


def plan(keep, add, held, table, free, max_rows, T):
    """The definition, sequence by sequence, on lists; returns what kv4_plan leaves."""
    held, table, free = list(held), [list(r) for r in table], list(free)
    n, blocks = len(keep), len(table[0])
    need = [-(-(k + a) // T) for k, a in zip(keep, add)]
    status, rows = [0] * n, 0
    for i in range(n):
        if keep[i] < 0 or add[i] < 0 or held[i] < 0 or keep[i] > held[i] * T or need[i] > blocks:
            status[i] = 2
            continue
        rows += add[i]
        if rows > max_rows:
            status[i] = 3
    for i in reversed(range(n)):
        if status[i] == 0:
            while held[i] > need[i]:
                held[i] -= 1
                free[0] += 1
                free[free[0]] = table[i][held[i]]
                table[i][held[i]] = -1
    count, want, start, slots, positions = free[0], 0, [0], [], []
    for i in range(n):
        if status[i] == 0 and need[i] > held[i]:
            want += need[i] - held[i]
            if want > count:
                status[i] = 1
            else:
                while held[i] < need[i]:
                    table[i][held[i]] = free[free[0]]
                    free[0] -= 1
                    held[i] += 1
        if status[i] == 0:
            for p in range(keep[i], keep[i] + add[i]):
                slots.append(table[i][p // T] * T + p % T)
                positions.append(p)
        start.append(len(slots))
    tail = [-1] * (max_rows - len(slots))
    return dict(held=held, table=table, free=free, row_start=start, slots=slots + tail, positions=positions + tail, status=status)


def attend(q, k, v, see, scale, kind):
    """One sequence: q [rows][hq][hd], k, v [keys][heads][hd] float64, see [rows][keys].  Returns (out, tolerance).

    What may differ, relative to half a step u of fp32: a score is a sum of hd exact products in fp32, each partial sum rounded: (hd + 4) u sum |q k| scale at
    most; its scaling, the subtraction of the maximum and the exponential: 4 u (|score| + 2) each.  A weight is off by twice the largest of these (its
    own, and the denominator's), plus the rounding to the operand type of the value product (bf16 queries: one step of bf16; fp32 ones: none, three
    parts hold 24 bits); the weighted sum adds (keys + 8) u of sum w |v|, the result its own type's rounding."""
    rows, hq, hd = q.shape
    heads, group = k.shape[1], hq // k.shape[1]
    u = U["float32"]
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(hq):
        kh, vh = k[:, h // group], v[:, h // group]
        for i in range(rows):
            on = see[i]
            if not on.any():
                continue
            s = kh[on] @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vh[on]
            size = np.abs(vh[on])
            off = (hd + 4) * u * (np.abs(kh[on]) @ np.abs(q[i, h])).max() * abs(scale) + 4 * u * (np.abs(s).max() + 2)
            weight = 2 * off + (U["bfloat16"] if kind == "bfloat16" else 0) + (on.sum() + 8) * u
            tol[i, h] = weight * (w @ size) + U[kind] * np.abs(out[i, h])
    return out, tol


def logprobs(x, tokens, temperature, top):
    """x [rows][vocab] float64; returns logprob, entropy, top ids, top logprobs"""
    y = x / temperature
    with np.errstate(all="ignore"):
        m = y.max(-1, keepdims=True)
        good = np.isfinite(m[:, 0]) & ~np.isnan(y).any(-1)
        e = np.exp(y - m)
        z = e.sum(-1, keepdims=True)
        lp = y - m - np.log(z)
        h = np.log(z[:, 0]) - np.where(e > 0, e * np.where(e > 0, y - m, 0), 0).sum(-1) / z[:, 0]
    inside = (tokens >= 0) & (tokens < x.shape[1])
    given = np.where(inside & good[:, None], np.take_along_axis(lp, np.clip(tokens, 0, x.shape[1] - 1), 1), np.nan)
    ids = np.argsort(-np.where(np.isnan(x), -np.inf, x), axis=-1, kind="stable")[:, :top]
    top_lp = np.where(good[:, None], np.take_along_axis(lp, ids, 1), np.nan)
    return given, np.where(good, h, np.nan), np.where(good[:, None], ids, -1), top_lp
