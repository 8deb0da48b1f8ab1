"""64-bit oracle of the calls on the caller's own memory: 4-bit pages, rows appended to paged caches, attention over them,
cross attention.  numpy, written from the formulas in include/nfd.h; shares nothing with the library.

A batch is a dict(rows=[...], lens=[...]): rows and tokens (keys) of every sequence; its rows lie one sequence behind the
other in the row buffers.
"""
import numpy as np


# ---- 4-bit numbers -------------------------------------------------------------------------------------------
def kv4_quantise(x):
    """x [..., dh] (fp32 values) -> whole numbers n [..., dh], z and step [..., dh / 32] (64 bits; step NaN: not finite)."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, 32))
    lo, hi = np.minimum(g.min(-1), 0.0), np.maximum(g.max(-1), 0.0)
    ok = np.isfinite(g).all(-1)
    # r >= hi - lo as r - big >= small: a difference that 64 bits hold, r being a number of few bits that is not far from big (or far above)
    big, small = np.where(ok, np.maximum(hi, -lo), 0.0), np.where(ok, np.minimum(hi, -lo), 0.0)
    ok &= float(np.finfo(np.float32).max) - big >= small
    big, small = np.where(ok, big, 0.0), np.where(ok, small, 0.0)
    up = lambda y: (lambda m, e: np.ldexp(np.ceil(m * 16) / 16, e))(*np.frexp(y))
    step = np.maximum(up((big + small) / 15), 2.0 ** -100)
    step = np.where(15 * step - big >= small, step, up(step * (1 + 2.0 ** -20)))
    g, lo = np.where(ok[..., None], g, 0.0), np.where(ok, lo, 0.0)
    z = np.rint(-lo / step)
    n = np.clip(np.rint(g / step[..., None]) + z[..., None], 0, 15)
    n = np.where(ok[..., None], n, 0).astype(np.int64).reshape(x.shape)
    return n, np.where(ok, z, 0).astype(np.int64), np.where(ok, step, np.nan)


def kv4_bytes(n, z, step):
    """The page's bytes [..., dh / 2] and words [..., dh / 32]."""
    e = n.reshape(n.shape[:-1] + (-1, 8))
    w = sum(e[..., i] << (4 * (i // 2) + 16 * (i % 2)) for i in range(8)).astype("<u4")
    bits = np.where(np.isnan(step), np.float32(np.nan), step).astype(np.float32).view(np.uint32) >> 16
    bits = np.where(np.isnan(step), 0x7FC0, bits)
    return w.view(np.uint8).reshape(n.shape[:-1] + (-1,)), ((bits & 0xFFF0) | z).astype(np.uint16)


def kv4_values(by, words):
    """What bytes and words stand for, 64 bits."""
    w = np.ascontiguousarray(by).view("<u4").astype(np.int64)
    n = np.stack([w >> (4 * (i // 2) + 16 * (i % 2)) & 15 for i in range(8)], -1).reshape(by.shape[:-1] + (by.shape[-1] // 16, 32))
    words = words.astype(np.uint32)
    step = ((words & 0xFFF0) << 16).astype(np.uint32).view(np.float32).astype(np.float64)
    return ((n - (words & 15).astype(np.int64)[..., None]) * step[..., None]).reshape(by.shape[:-1] + (2 * by.shape[-1],))


# ---- rotation ------------------------------------------------------------------------------------------------
def rotate(x, positions, rope, theta, frame_tokens, grid_w):
    """x [n, H, dh] fp32 -> fp32: angles in 64 bits, sines and cosines rounded to fp32, the rotation's four products and two
    sums rounded to fp32 each."""
    x, p = np.asarray(x, np.float32), np.asarray(positions, np.int64)
    axes = (p // frame_tokens, p % frame_tokens // grid_w, p % frame_tokens % grid_w)
    th = float(np.float32(theta))
    a = np.concatenate([axes[i][:, None] * th ** (-2.0 * np.arange(d // 2) / max(d, 1)) for i, d in enumerate(rope)], 1)
    c, s = np.cos(a).astype(np.float32)[:, None], np.sin(a).astype(np.float32)[:, None]
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return np.stack([x0 * c - x1 * s, x1 * c + x0 * s], -1).reshape(x.shape)


# ---- places --------------------------------------------------------------------------------------------------
def place(table_row, token, page_tokens):
    """(page, offset) of a token; the table is a ring."""
    return int(table_row[(token // page_tokens) % len(table_row)]), token % page_tokens


def held_from(n_tokens, table_len, page_tokens):
    """The first token that a ring has not overwritten."""
    return max(0, n_tokens - table_len * page_tokens)


# ---- attention -----------------------------------------------------------------------------------------------
def attend(q, k, v, seen):
    """One head: q [n, dh], k and v [L, dh], seen [n, L].  Returns the result and sum p |v| (for error bounds)."""
    n, dh = q.shape
    out, mag = np.zeros((n, dh)), np.zeros((n, dh))
    if k.shape[0] == 0:
        return out, mag
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.where(seen, q @ k.T / np.sqrt(dh), -np.inf)
        m = np.where(np.isneginf(s).all(1), 0.0, s.max(1, initial=-np.inf))
        p = np.exp(s - m[:, None])
    total = p.sum(1)
    p = p / np.where(total == 0, 1.0, total)[:, None]
    vis = seen.any(0)
    return p[:, vis] @ v[vis], p[:, vis] @ np.abs(v[vis])


def attention_kv4(q, batch, table, pages, frame_tokens, window, share):
    """q [n_rows, H, dh]; pages = (k bytes, k words, v bytes, v words) [pages, Hk, P, ..] -> (out, magnitude) [n_rows, H, dh]."""
    kb, kw, vb, vw = pages
    n_pages, _, page_tokens, _ = kb.shape
    out, mag, r0 = np.zeros(q.shape), np.zeros(q.shape), 0
    for s, (n, length) in enumerate(zip(batch["rows"], batch["lens"])):
        toks = [(t,) + place(table[s], t, page_tokens) for t in range(held_from(length, table.shape[1], page_tokens), length)]
        toks = [t for t in toks if 0 <= t[1] < n_pages]
        t, pg, off = (np.array([x[i] for x in toks], np.int64) for i in range(3))
        pos = length - n + np.arange(n)
        f = pos // frame_tokens
        seen = ((t[None] >= np.maximum(f - window, 0)[:, None] * frame_tokens)
                & (t[None] < ((f + 1) * frame_tokens)[:, None]) & (pos >= 0)[:, None])
        for h in range(q.shape[1]):
            g = h // share
            k, v = kv4_values(kb[pg, g, off], kw[pg, g, off]), kv4_values(vb[pg, g, off], vw[pg, g, off])
            out[r0:r0 + n, h], mag[r0:r0 + n, h] = attend(np.asarray(q[r0:r0 + n, h], np.float64), k, v, seen)
        r0 += n
    return out, mag


def cross_attention(q, batch, k, v, mask, share):
    """q [n_rows, H, dh], k and v [S, L, Hk, dh], mask [S, L] or None -> (out, magnitude) [n_rows, H, dh]."""
    out, mag, r0 = np.zeros(q.shape), np.zeros(q.shape), 0
    for s, (n, length) in enumerate(zip(batch["rows"], batch["lens"])):
        keep = np.arange(min(length, k.shape[1]))
        if mask is not None:
            keep = keep[mask[s, keep].astype(bool)]
        for h in range(q.shape[1]):
            kk, vv = np.asarray(k[s, keep, h // share], np.float64), np.asarray(v[s, keep, h // share], np.float64)
            out[r0:r0 + n, h], mag[r0:r0 + n, h] = attend(np.asarray(q[r0:r0 + n, h], np.float64), kk, vv,
                                                         np.ones((n, len(keep)), bool))
        r0 += n
    return out, mag
