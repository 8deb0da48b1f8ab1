"""The calls for hosts that bring their own memory, as timed cases beside their plain forms.

append   new rows of keys and values go into a paged cache, rotated on the way; the rows' queries are rotated with them.
         Pages hold fp32, bf16 or 4-bit numbers; rows that went into 4-bit pages are read back out of them.
kv4      attention over a cache of 4-bit pages: a batch of sequences, page tables, heads that share keys, the library's
         block-causal window (frames of one token: a causal one).
cross    attention of a batch of rows to the states of an encoder, of another length, with lengths and a mask of keys.

A 4-bit page holds, for 32 numbers of a row, whole numbers n of 4 bits and a 16-bit word: the upper 12 bits are those of a
bf16 step, the lower 4 a whole number z.  They stand for (n - z) step.  Eight numbers are a 32-bit word, the even ones in
its lower half, the odd ones in its upper half, each half with the first one lowest.
"""
import math

import torch

own = False

DEV = "cuda:0"
THETA = 10000.0
ROPE3 = {32: (8, 12, 12), 64: (16, 24, 24), 128: (32, 48, 48)}      # frame, row and column shares of the head dimension
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _append(dtype, pages, seqs, rows, heads, kv_heads, head_dim, page, frame, grid_w, ctx, ragged=False):
    return dict(op="append", dtype=dtype, pages=pages, seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, page=page, frame=frame, grid_w=grid_w, ctx=ctx, ragged=ragged)


def _kv4(seqs, rows, heads, kv_heads, head_dim, page, frame, window, ctx, ragged=False):
    return dict(op="kv4", seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, frame=frame,
                window=window, ctx=ctx, ragged=ragged)


def _cross(dtype, seqs, rows, heads, kv_heads, head_dim, keys, ragged=False, mask=False):
    return dict(op="cross", dtype=dtype, seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                keys=keys, ragged=ragged, mask=mask)


def listed():
    return [
        # a server's step of eight sequences, one token each, into small pages
        dict(name="append_tokens8", **_append("bf16", "bf16", 8, 1, 16, 16, 64, 16, 1, 1, 2000)),
        # the 310M-class model's next frame into its frame page, behind 16 others
        dict(name="append_frame", **_append("bf16", "bf16", 1, 336, 16, 16, 64, 336, 336, 14, 17 * 336)),
        # eight streams of that model, four speculative frames each, into a 4-bit cache, and read back
        dict(name="append_kv4_streams8", **_append("bf16", "int4", 8, 4 * 336, 16, 16, 64, 336, 336, 14, 33 * 336)),
        # a small fp32 model at an odd size, pages that end inside a frame, one sequence without rows
        dict(name="append_fp32_odd", **_append("fp32", "fp32", 3, 77, 6, 6, 32, 50, 77, 7, 700, True)),
        # one token behind the 310M-class model's window of 17 frames
        dict(name="kv4_token", **_kv4(1, 1, 16, 16, 64, 336, 1, 1 << 30, 17 * 336)),
        # eight long sequences of different lengths, one token each, three heads to a pair of keys and values
        dict(name="kv4_tokens8_shared", **_kv4(8, 1, 24, 8, 128, 64, 1, 1 << 30, 32768, True)),
        # the 310M-class model's next frame behind 16 frames: the headline's attention on a 4-bit cache
        dict(name="kv4_frame", **_kv4(1, 336, 16, 16, 64, 336, 336, 16, 17 * 336)),
        # a server: eight streams behind 32 frames
        dict(name="kv4_streams8", **_kv4(8, 336, 16, 16, 64, 336, 336, 32, 33 * 336)),
        # one row of eight sequences each against a short encoded prompt
        dict(name="cross_rows8", **_cross("bf16", 8, 1, 16, 16, 64, 77)),
        # a frame of the 310M-class model against an encoded prompt with padding in places
        dict(name="cross_frame", **_cross("bf16", 1, 336, 16, 16, 64, 512, False, True)),
        # four frames of eight streams against long encoded sequences, four heads to a pair
        dict(name="cross_streams8", **_cross("bf16", 8, 4 * 336, 16, 4, 128, 2048, True)),
        # the small fp32 model
        dict(name="cross_fp32_odd", **_cross("fp32", 3, 77, 6, 6, 32, 220, True)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(4, 4, 32), (6, 6, 32), (12, 12, 64), (16, 16, 64), (24, 24, 64), (8, 2, 64), (16, 4, 128), (24, 8, 128), (8, 1, 128)]
FRAMES = [(336, 14), (220, 11), (77, 7), (64, 8), (1, 1)]


def _draw(rng):
    heads, kv_heads, head_dim = rng.choice(HEADS)
    seqs, ragged = _log_int(rng, 1, 12), rng.random() < 0.4
    op = rng.choice(["append", "kv4", "cross"])
    few = rng.random() < 0.4
    rows = rng.randint(1, 4) if few else _log_int(rng, 5, 1400)
    if op == "cross":
        dtype = "fp32" if rng.random() < 0.15 else "bf16"
        return _cross(dtype, seqs, rows, heads, kv_heads, head_dim, _log_int(rng, 1, 4096), ragged, rng.random() < 0.4)
    frame, grid_w = rng.choice(FRAMES)
    page = rng.choice([frame, 16, 50, 64, 128]) if frame > 1 else rng.choice([16, 50, 64, 128, 336])
    if op == "append":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        pages = rng.choice([dtype, "int4"])
        return _append(dtype, pages, seqs, rows, heads, kv_heads, head_dim, page, frame, grid_w,
                       rows + _log_int(rng, 1, 20000), ragged)
    window = rng.randint(1, 32) if frame > 1 else rng.choice([1 << 30, 1 << 30, _log_int(rng, 64, 4096)])
    return _kv4(seqs, rows, heads, kv_heads, head_dim, page, frame, window, rows + _log_int(rng, 1, 32768 if few else 11000),
                ragged)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


def _sizes(case):
    """Rows and tokens (keys) of every sequence: a rule, so that work() knows them too."""
    n, r = case["seqs"], case["rows"]
    total = case["keys"] if case["op"] == "cross" else case["ctx"]
    if not case["ragged"]:
        return [r] * n, [total] * n
    rows = [0 if s == 2 else max(1, r - (s * 13 % 5) * r // 6) for s in range(n)]
    lens = [max(0 if case["op"] == "cross" and s == 1 else 1, total - (s * 29 % 7) * total // 9) for s in range(n)]
    return rows, lens if case["op"] == "cross" else [max(a, b) for a, b in zip(lens, rows)]


def _first_key(case, rows, length):
    """The first token that any of a sequence's rows sees."""
    return max(0, (length - rows) // case["frame"] - case["window"]) * case["frame"]


def work(case):
    rows, lens = _sizes(case)
    h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    size = 4 if case.get("dtype") == "fp32" else 2
    n = sum(rows)
    if case["op"] == "append":
        per = {"fp32": 4, "bf16": 2, "int4": 0.5 + 2 / 32}[case["pages"]]
        moved = n * dh * (2 * h * size + 2 * hk * (size + per))
        back = 2 * n * hk * dh * 2 if case["pages"] == "int4" else 0       # the rows read back, as bf16
        return {"bytes": moved + back, "flops": n * dh * (h + hk) * 3}
    if case["op"] == "kv4":
        keys = pairs = 0
        for r, l in zip(rows, lens):
            keys += l - _first_key(case, r, l) if r else 0
            f = case["frame"]
            p, end, at = l - r, l, 0
            while p < end:                                                 # the rows of one frame see the same keys
                stop = min(end, (p // f + 1) * f)
                at += (stop - p) * (min(end, (p // f + 1) * f) - max(0, p // f - case["window"]) * f)
                p = stop
            pairs += at
        return {"bytes": 2 * keys * hk * dh * (0.5 + 2 / 32) + 4 * n * h * dh, "flops": 4 * pairs * h * dh}
    keys = sum(l for r, l in zip(rows, lens) if r)
    return {"bytes": size * (2 * keys * hk * dh + 2 * n * h * dh), "flops": 4 * sum(r * l for r, l in zip(rows, lens)) * h * dh}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---------------------------------------------------------------------------------------------------------------
# state
# ---------------------------------------------------------------------------------------------------------------
def _randn(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _rows(case):
    """What says which rows belong to which sequence: row_start, kv_len and for each place of a [seqs, most rows] table the row."""
    rows, lens = _sizes(case)
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    n = start[-1] + (3 if case["ragged"] else 0)               # rows behind the last sequence, as in a padded batch
    most = max(rows)
    i = torch.arange(most, device=DEV)
    count = torch.tensor(rows, device=DEV)
    row_start = torch.tensor(start, device=DEV, dtype=torch.int32)
    return dict(n_rows=n, max_rows=most, row_start=row_start, kv_len=torch.tensor(lens, device=DEV, dtype=torch.int32),
                valid=i[None] < count[:, None], index=row_start[:-1, None].long() + i[None],
                position=(torch.tensor(lens, device=DEV) - count)[:, None] + i[None])


def _pool(case, gen, state):
    """Page pools with the cached tokens of every sequence in pages that lie in no order, and the page table."""
    n, hk, dh, p = case["seqs"], case["kv_heads"], case["head_dim"], case["page"]
    per = -(-case["ctx"] // p)
    state["table"] = torch.randperm(n * per, generator=gen, device=DEV).view(n, per).int()
    kind = "int4" if case["op"] == "kv4" else case["pages"]
    for name in ("k", "v"):
        x = _randn(gen, n * per, hk, p, dh)
        if name == "k":                                        # keys have channels that are larger than the others
            x = x * (1 + 3 * (torch.arange(dh, device=DEV) % 16 == 5))
        if kind == "int4":
            state[name], state[name + "_scale"] = _quantise(x)
        else:
            state[name], state[name + "_scale"] = x.to(TYPES[kind]), None


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    dtype = TYPES[case.get("dtype", "bf16")]
    h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    s = dict(case=case, **_rows(case))
    n = s["n_rows"]
    if case["op"] == "append":
        _pool(case, gen, s)
        qkv = _randn(gen, n, (h + 2 * hk) * dh, dtype=dtype)    # the projection's output; its parts are taken as they lie
        q, k, v = qkv.split([h * dh, hk * dh, hk * dh], dim=1)
        s.update(q=q.unflatten(1, (h, dh)), new_k=k.unflatten(1, (hk, dh)), new_v=v.unflatten(1, (hk, dh)),
                 q_out=torch.zeros(n, h, dh, device=DEV, dtype=dtype))
        s["rope"] = ROPE3[dh] if case["frame"] > 1 else (dh, 0, 0)
        if case["pages"] == "int4":
            s.update(k_rows=torch.zeros(n, hk, dh, device=DEV, dtype=torch.bfloat16),
                     v_rows=torch.zeros(n, hk, dh, device=DEV, dtype=torch.bfloat16))
    else:
        s["q"] = _randn(gen, n, h, dh, dtype=dtype)
        s["out"] = torch.zeros(n, h * dh, device=DEV, dtype=dtype)
        if case["op"] == "kv4":
            _pool(case, gen, s)
            rows, lens = _sizes(case)
            first = [_first_key(case, r, l) for r, l in zip(rows, lens)]
            s["first"] = torch.tensor(first, device=DEV)
            s["span"] = max(l - f for l, f in zip(lens, first))
        else:
            kv = _randn(gen, case["seqs"], case["keys"], 2, hk, dh, dtype=dtype)
            s["mask"] = None
            if case["mask"]:
                s["mask"] = torch.rand(case["seqs"], case["keys"], generator=gen, device=DEV) < 0.8
            if case["ragged"]:                                 # what lies behind a sequence's end is not to be looked at
                beyond = torch.arange(case["keys"], device=DEV)[None] >= s["kv_len"][:, None]
                kv[beyond] = float("nan")
            s.update(enc_k=kv[:, :, 0], enc_v=kv[:, :, 1])
    if own:
        from paper_2506_01380_b200 import nfd as N
        s["batch"] = N.Batch(n, s["kv_len"], table=s.get("table"), row_start=s["row_start"], max_rows=s["max_rows"])
        if case["op"] == "cross":
            s["states"] = N.States(s["enc_k"], s["enc_v"], mask=s["mask"])
        else:
            s["pages"] = N.Pages(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if case["op"] == "append":
            s["rotation"] = N.Rope(*s["rope"], theta=THETA, frame_tokens=case["frame"], grid_w=case["grid_w"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _quantise(x):
    """fp32 [..., dh] -> 4-bit numbers [..., dh / 2] uint8 and words [..., dh / 32] int16."""
    g = x.unflatten(-1, (-1, 32))
    lo, hi = g.amin(-1).clamp(max=0), g.amax(-1).clamp(min=0)
    # (in 64 bits: a number half way between two steps, which bf16 inputs often are, goes to the even one)
    top = (hi - lo).double().div(15).clamp(min=2.0 ** -100).view(torch.int64)
    step = (top + ((1 << 49) - 1) & ~((1 << 49) - 1)).view(torch.float64)            # up to the next number of 4 bits
    bits = step.float().view(torch.int32)
    z = torch.round(-lo / step)
    n = (torch.round(g / step[..., None]) + z[..., None]).clamp(0, 15).to(torch.int32).flatten(-2)
    word = (bits >> 16) | z.to(torch.int32)
    e = n.unflatten(-1, (-1, 8))
    half = lambda a: a[..., 0] | a[..., 1] << 4 | a[..., 2] << 8 | a[..., 3] << 12
    low, high = half(e[..., 0::2]), half(e[..., 1::2])
    packed = torch.stack([low & 255, low >> 8, high & 255, high >> 8], -1).flatten(-2)
    return packed.to(torch.uint8), word.to(torch.int16)


def _dequantise(packed, word):
    """The numbers, fp32, that codes [..., dh / 2] and words [..., dh / 32] stand for."""
    b = packed.unflatten(-1, (-1, 4)).to(torch.int32)
    low, high = b[..., 0] | b[..., 1] << 8, b[..., 2] | b[..., 3] << 8
    shift = torch.tensor([0, 4, 8, 12], device=packed.device, dtype=torch.int32)
    n = torch.stack([low[..., None] >> shift & 15, high[..., None] >> shift & 15], -1)
    w = word.to(torch.int32)
    step = (w << 16 & -0x100000).view(torch.float32)
    n = n.flatten(-3).unflatten(-1, (-1, 32))
    return ((n - (w & 15)[..., None]).float() * step[..., None]).flatten(-2)


def _angles(case, rope, position):
    """cos and sin [rows, dh / 2], fp32, of a row's pairs: angles in 64 bits."""
    f, gw = case["frame"], case["grid_w"]
    axes = [position // f, position % f // gw, position % f % gw]
    parts = [axes[i].double()[:, None] * THETA ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / max(d, 1))
             for i, d in enumerate(rope)]
    a = torch.cat(parts, 1)
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _rotate(x, cos, sin):
    x0, x1 = x[..., 0::2].float(), x[..., 1::2].float()
    return torch.stack([x0 * cos - x1 * sin, x1 * cos + x0 * sin], -1).flatten(-2)


def _run_append(s):
    case = s["case"]
    at, pos = s["index"][s["valid"]], s["position"][s["valid"]]
    seq = torch.arange(case["seqs"], device=DEV)[:, None].expand_as(s["valid"])[s["valid"]]
    page, off = s["table"][seq, pos // case["page"]].long(), pos % case["page"]
    cos, sin = _angles(case, s["rope"], pos)
    s["q_out"][at] = _rotate(s["q"][at], cos, sin).to(s["q_out"].dtype)
    k, v = _rotate(s["new_k"][at], cos, sin), s["new_v"][at].float()
    if case["pages"] != "int4":
        s["k"][page, :, off] = k.to(s["k"].dtype)
        s["v"][page, :, off] = v.to(s["v"].dtype)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    kc, kw = _quantise(k)
    vc, vw = _quantise(v)
    s["k"][page, :, off], s["k_scale"][page, :, off] = kc, kw
    s["v"][page, :, off], s["v_scale"][page, :, off] = vc, vw
    s["k_rows"][at] = _dequantise(s["k"][page, :, off], s["k_scale"][page, :, off]).to(torch.bfloat16)
    s["v_rows"][at] = _dequantise(s["v"][page, :, off], s["v_scale"][page, :, off]).to(torch.bfloat16)
    return {"q": s["q_out"], "k": s["k_rows"], "v": s["v_rows"]}


def _softmax_attention(s, q, k, v, seen):
    """q [B, R, H, dh], k and v [B, L, Hk, dh] fp32, seen [B, R or 1, L]; the rows' results go where they belong."""
    b, r, h, dh = q.shape
    hk = k.shape[2]
    q = q.view(b, r, hk, h // hk, dh).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, dh)          # [B, Hk, heads of the pair x R, dh]
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) * (1 / math.sqrt(dh))
    x = x.view(b, h, r, -1).masked_fill_(~seen[:, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x.sub_(torch.where(m == float("-inf"), 0.0, m)))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, p.shape[-1]), v.transpose(1, 2)).view(b, h, r, dh)
    o = o / torch.where(total == 0, 1.0, total)
    out = torch.zeros_like(s["out"])
    out[s["index"][s["valid"]]] = o.transpose(1, 2)[s["valid"]].flatten(1).to(out.dtype)
    return out


def _padded_q(s):
    return s["q"][s["index"].clamp(max=s["n_rows"] - 1)].float()


def _run_kv4(s):
    case = s["case"]
    pos = s["first"][:, None] + torch.arange(s["span"], device=DEV)[None]                    # [B, L]
    page = s["table"].gather(1, (pos // case["page"]).clamp(max=s["table"].shape[1] - 1)).long()
    off = pos % case["page"]
    k = _dequantise(s["k"][page, :, off], s["k_scale"][page, :, off])
    v = _dequantise(s["v"][page, :, off], s["v_scale"][page, :, off])
    frame = s["position"] // case["frame"]                                                    # [B, R]
    lo = (frame - case["window"]).clamp(min=0) * case["frame"]
    hi = torch.minimum((frame + 1) * case["frame"], s["kv_len"][:, None])
    seen = (pos[:, None] >= lo[..., None]) & (pos[:, None] < hi[..., None])
    return _softmax_attention(s, _padded_q(s), k, v, seen)


def _run_cross(s):
    k, v = s["enc_k"].float(), s["enc_v"].float()
    seen = torch.arange(k.shape[1], device=DEV)[None] < s["kv_len"][:, None]
    if s["mask"] is not None:
        seen = seen & s["mask"]
    return _softmax_attention(s, _padded_q(s), k, v.masked_fill(~seen[:, :, None, None], 0.0), seen[:, None])


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"append": _run_append, "kv4": _run_kv4, "cross": _run_cross}[op](s)
    from paper_2506_01380_b200 import nfd as N
    if op == "kv4":
        return N.attention_kv4(s["pages"], s["batch"], s["q"], s["out"], frame_tokens=s["case"]["frame"],
                               window=s["case"]["window"])
    if op == "cross":
        return N.cross_attention(s["states"], s["batch"], s["q"], s["out"])
    N.kv_append(s["pages"], s["batch"], s["new_k"], s["new_v"], s["rotation"], q=s["q"], q_out=s["q_out"])
    if s["case"]["pages"] != "int4":
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    N.pages_read(s["pages"], s["batch"], s["k_rows"], s["v_rows"])
    return {"q": s["q_out"], "k": s["k_rows"], "v": s["v_rows"]}


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------------------------------------------
def _values64(codes, words):
    """Numbers of 4-bit rows [..., dh / 2], [..., dh / 32], from their definition: number by number of a 32-bit word."""
    by = codes.long().unflatten(-1, (-1, 4))
    whole = by[..., 0] + by[..., 1] * 256 + by[..., 2] * 65536 + by[..., 3] * 16777216
    n = torch.stack([whole // 16 ** (i // 2 + 4 * (i % 2)) % 16 for i in range(8)], -1).flatten(-2)
    w = words.long() % 65536
    e, frac = w // 128, w // 16 % 8
    step = (1 + frac.double() / 8) * torch.pow(2.0, e.double() - 127)
    return ((n.unflatten(-1, (-1, 32)) - (w % 16)[..., None]).double() * step[..., None]).flatten(-2)


def _held64(x):
    """What 4-bit pages hold for rows of x (64 bits)."""
    g = x.unflatten(-1, (-1, 32))
    lo, hi = torch.minimum(g.amin(-1), torch.zeros_like(g[..., 0])), torch.maximum(g.amax(-1), torch.zeros_like(g[..., 0]))
    mant, ex = torch.frexp((hi - lo) / 15)                      # mant in [0.5, 1)
    step = torch.ldexp(torch.ceil(mant * 16) / 16, ex).clamp(min=2.0 ** -100)[..., None]
    z = torch.round(-lo[..., None] / step)
    return (((torch.round(g / step) + z).clamp(0, 15) - z) * step).flatten(-2)


def _turned64(x, case, rope, position):
    z = torch.view_as_complex(x.double().unflatten(-1, (-1, 2)).contiguous())
    f = case["frame"]
    at = (position // f, position % f // case["grid_w"], position % f % case["grid_w"])
    angle = [at[a].double() * THETA ** (-2.0 * i / d) for a, d in enumerate(rope) for i in range(d // 2)]
    a = torch.stack(angle, -1)[:, None]
    return torch.view_as_real(z * torch.polar(torch.ones_like(a), a)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    rows, lens = _sizes(case)
    h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    start = s["row_start"].tolist()
    if case["op"] == "append":
        held = _held64 if case["pages"] == "int4" else (lambda x: x)
        q = s["q_out"].double()
        if case["pages"] == "int4":
            k, v = s["k_rows"].double(), s["v_rows"].double()
        else:
            k, v = s["k"].double(), s["v"].double()
        for b, (r, l) in enumerate(zip(rows, lens)):
            if not r:
                continue
            here = slice(start[b], start[b] + r)
            pos = torch.arange(l - r, l, device=DEV)
            q[here] = _turned64(s["q"][here], case, s["rope"], pos)
            nk, nv = held(_turned64(s["new_k"][here], case, s["rope"], pos)), held(s["new_v"][here].double())
            if case["pages"] == "int4":
                k[here], v[here] = nk, nv
            else:
                page = s["table"][b].long()[pos // case["page"]]
                k[page, :, pos % case["page"]], v[page, :, pos % case["page"]] = nk, nv
        return {"q": q, "k": k, "v": v}
    out = torch.zeros(s["n_rows"], h, dh, device=DEV, dtype=torch.float64)
    for b, (r, l) in enumerate(zip(rows, lens)):
        if not r:
            continue
        if case["op"] == "kv4":
            first = _first_key(case, r, l)
            pos = torch.arange(first, l, device=DEV)
            page, off = s["table"][b].long()[pos // case["page"]], pos % case["page"]
            k = _values64(s["k"][page, :, off], s["k_scale"][page, :, off])
            v = _values64(s["v"][page, :, off], s["v_scale"][page, :, off])
            fq, fk = torch.arange(l - r, l, device=DEV) // case["frame"], pos // case["frame"]
            hidden = (fk[None] > fq[:, None]) | (fk[None] < fq[:, None] - case["window"])
        else:
            keep = torch.arange(l, device=DEV)
            if s["mask"] is not None:
                keep = keep[s["mask"][b, :l]]
            k, v = s["enc_k"][b, keep].double(), s["enc_v"][b, keep].double()
            hidden = torch.zeros(r, len(keep), device=DEV, dtype=torch.bool)
        if not k.shape[0]:
            continue
        for head in range(h):
            g = head * hk // h
            x = s["q"][start[b]:start[b] + r, head].double() @ k[:, g].T / math.sqrt(dh)
            x = torch.where(hidden, torch.full_like(x, float("-inf")), x)
            out[start[b]:start[b] + r, head] = torch.exp(x - torch.logsumexp(x, 1, keepdim=True)) @ v[:, g]
    return out.flatten(1)
