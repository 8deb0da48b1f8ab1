"""64-bit oracle of the calls around a block's projections: attention over pages and over packed prompts, rotation, norms with gate
and residual.  torch in float64 on whatever device the inputs are, written from the formulas in include/nfd.h; shares nothing with
the library.
"""
import math

import torch


def seen_tokens(n, length, frame_tokens, window, oldest=0):
    """bool [n, length]: what the last n of `length` tokens see (rows of tokens below 0: nothing)."""
    pos = torch.arange(length - n, length)
    f = torch.div(pos, frame_tokens, rounding_mode="floor")
    t = torch.arange(length)
    lo, hi = (f - window).clamp(min=0) * frame_tokens, (f + 1) * frame_tokens
    return (t[None] >= lo[:, None]) & (t[None] < hi[:, None]) & (pos >= 0)[:, None] & (t >= oldest)[None]


def attend(q, k, v, seen):
    """q [n, H, dh], k and v [L, Hk, dh], seen [n, L].  Returns (out, sum p |v|), [n, H, dh]: what no row sees counts for nothing,
    whatever it is; a value that is not finite makes its column of the rows that see it so."""
    n, h, dh = q.shape
    share = h // k.shape[1]
    out, mag = (torch.zeros(n, h, dh, dtype=torch.float64, device=q.device) for _ in range(2))
    if k.shape[0] == 0 or n == 0:
        return out, mag
    seen = seen.to(q.device)
    late = ~torch.isfinite(v.double())
    val = torch.where(late, 0.0, v.double())
    for i in range(h):
        g = i // share
        s = (q[:, i].double() @ k[:, g].double().T / math.sqrt(dh)).masked_fill(~seen, -math.inf)
        m = s.amax(1, keepdim=True)
        p = torch.exp(s - torch.where(torch.isneginf(m), 0.0, m))
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
        out[:, i], mag[:, i] = p @ val[:, g], p @ val[:, g].abs()
        if late[:, g].any():
            out[:, i] += torch.where((seen.double() @ late[:, g].double()) > 0, math.nan, 0.0)
    return out, mag


def rotate(x, positions, rope, theta, halves=False, back=False):
    """x [n, H, dh], positions [n, 3] -> float64."""
    x, p = x.double(), positions.double()
    freq = [(a, float(theta) ** (-2.0 * i / d)) for a, d in enumerate(rope) for i in range(d // 2)]
    angle = torch.stack([p[:, a] * f for a, f in freq], 1)[:, None]
    c, s = torch.cos(angle), torch.sin(angle) * (-1 if back else 1)
    a, b = x.chunk(2, -1) if halves else (x[..., 0::2], x[..., 1::2])
    u, w = a * c - b * s, b * c + a * s
    return torch.cat([u, w], -1) if halves else torch.stack([u, w], -1).flatten(-2)


def normed(x, kind, eps, weight=None, bias=None):
    x = x.double()
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    x = x * weight.double() if weight is not None else x
    return x + bias.double() if bias is not None else x


def gate_norm(x, y, post, pre, gate, scale, shift, res_scale):
    """post, pre: (kind, eps, weight, bias) or None; gate, scale, shift [n, width] (a row's own) or None -> (x_out, h)."""
    x = x.double()
    if y is not None:
        t = normed(y, *post) if post is not None else y.double()
        x = x + res_scale * (t * gate.double() if gate is not None else t)
    h = None
    if pre is not None:
        h = normed(x, *pre)
        h = h * (1 + scale.double()) if scale is not None else h
        h = h + shift.double() if shift is not None else h
    return x, h
