"""What a host with its own memory needs to run a block of a transformer around its projections, as timed cases beside the plain forms.

pages    attention of a chunk of new rows over a paged cache of bf16 or fp32 numbers: a batch of sequences, page tables, heads
         that share keys, the library's block-causal window (frames of one token: a causal one); from single tokens to frames.
packed   attention over whole prompts: sequences of different lengths one behind the other, whose rows are queries, keys and
         values, causal or block-causal, heads that share keys.
rotate   rotary embedding of rows of queries and keys with a position on several axes (time, height, width) for each row.
norm     x' = x + a gate * post(y), h = pre(x') (1 + scale) + shift: the norms around a block, its gate and its residual scale.
"""
import math

import torch

own = False

DEV = "cuda:0"
THETA = 10000.0
EPS = 1e-6
ROPE3 = {32: (8, 12, 12), 64: (16, 24, 24), 128: (32, 48, 48)}      # frame, row and column shares of the head dimension
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _pages(dtype, seqs, rows, heads, kv_heads, head_dim, page, frame, window, ctx, ragged=False):
    return dict(op="pages", dtype=dtype, seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page,
                frame=frame, window=window, ctx=ctx, ragged=ragged)


def _packed(dtype, seqs, rows, heads, kv_heads, head_dim, frame, window, ragged=False):
    return dict(op="packed", dtype=dtype, seqs=seqs, rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                frame=frame, window=window, ragged=ragged)


def _rotary(dtype, rows, heads, kv_heads, head_dim, frame, grid_w, halves=False, in_place=False):
    return dict(op="rotate", dtype=dtype, rows=rows, heads=heads, kv_heads=kv_heads, head_dim=head_dim, frame=frame,
                grid_w=grid_w, halves=halves, in_place=in_place)


def _norm(x_type, dtype, rows, width, frames, kind, post=False, first=False):
    return dict(op="norm", x_type=x_type, dtype=dtype, rows=rows, width=width, frames=frames, kind=kind, post=post, first=first)


EVER = 1 << 30


def listed():
    return [
        # one token behind the 310M-class model's window of 17 frames
        dict(name="pages_token", **_pages("bf16", 1, 1, 16, 16, 64, 336, 1, EVER, 17 * 336)),
        # a server's step: sixteen sequences of different lengths, one token each, three heads to a pair of keys and values
        dict(name="pages_tokens16_shared", **_pages("bf16", 16, 1, 24, 8, 128, 64, 1, EVER, 16384, True)),
        # four long sequences, each with a chunk of 512 new tokens, four heads to a pair, small pages
        dict(name="pages_chunks4", **_pages("bf16", 4, 512, 16, 4, 128, 64, 1, EVER, 16384)),
        # eight streams of the 310M-class model, a frame each behind 32 frames: the served batch's attention
        dict(name="pages_streams8", **_pages("bf16", 8, 336, 16, 16, 64, 336, 336, 32, 33 * 336)),
        # a small fp32 model at an odd size, pages that end inside a frame, one sequence without rows
        dict(name="pages_fp32_odd", **_pages("fp32", 3, 77, 6, 6, 32, 50, 77, 7, 700, True)),
        # short encoded prompts of different lengths, packed one behind the other
        dict(name="packed_short", **_packed("bf16", 12, 200, 16, 16, 64, 1, EVER, True)),
        # long prompts of a model with four heads to a pair
        dict(name="packed_long", **_packed("bf16", 2, 8192, 16, 4, 128, 1, EVER)),
        # the first 16 frames of four streams of the 310M-class model, block-causal
        dict(name="packed_frames", **_packed("bf16", 4, 16 * 336, 16, 16, 64, 336, 16)),
        # a server's step of eight sequences, one token each
        dict(name="rotate_tokens8", **_rotary("bf16", 8, 16, 16, 64, 1, 1)),
        # the first 16 frames of four streams: positions in time, height and width, in place in the projection's output
        dict(name="rotate_video", **_rotary("bf16", 4 * 16 * 336, 16, 16, 64, 336, 14, False, True)),
        # between attention and MLP of a frame of the 310M-class model: gate, residual, norm, modulation
        dict(name="norm_frame", **_norm("fp32", "bf16", 336, 1024, 1, "layer")),
        # the same for the first 16 frames of four streams at the 774M-class width, with a norm behind the block as well
        dict(name="norm_video", **_norm("fp32", "bf16", 4 * 16 * 336, 1536, 64, "rms", True)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(4, 4, 32), (6, 6, 32), (12, 12, 64), (16, 16, 64), (24, 24, 64), (8, 2, 64), (16, 4, 128), (24, 8, 128), (8, 1, 128)]
FRAMES = [(336, 14), (220, 11), (77, 7), (64, 8), (1, 1)]


def _draw(rng):
    op = rng.choice(["pages", "pages", "packed", "packed", "rotate", "norm"])
    heads, kv_heads, head_dim = rng.choice(HEADS)
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    frame, grid_w = rng.choice(FRAMES)
    ragged = rng.random() < 0.4
    if op == "pages":
        few = rng.random() < 0.4
        rows = rng.randint(1, 4) if few else _log_int(rng, 5, 1400)
        page = rng.choice([frame, 16, 50, 64, 128]) if frame > 1 else rng.choice([16, 50, 64, 128, 336])
        window = rng.randint(1, 32) if frame > 1 else rng.choice([EVER, EVER, _log_int(rng, 64, 4096)])
        return _pages(dtype, _log_int(rng, 1, 16), rows, heads, kv_heads, head_dim, page, frame, window,
                      rows + _log_int(rng, 1, 20000), ragged)
    if op == "packed":
        window = rng.randint(1, 32) if frame > 1 else rng.choice([EVER, EVER, _log_int(rng, 64, 4096)])
        return _packed(dtype, _log_int(rng, 1, 16), _log_int(rng, 1, 8192), heads, kv_heads, head_dim, frame, window, ragged)
    if op == "rotate":
        return _rotary(dtype, _log_int(rng, 1, 20000), heads, kv_heads, head_dim, frame, grid_w, rng.random() < 0.5,
                       rng.random() < 0.5)
    width = rng.choice([128, 768, 1024, 1536, 2048, 4096, 8 * _log_int(rng, 8, 1000)])
    return _norm(rng.choice(["fp32", "fp32", "bf16"]), dtype, _log_int(rng, 1, 20000), width, _log_int(rng, 1, 64),
                 rng.choice(["layer", "rms"]), rng.random() < 0.4, rng.random() < 0.2)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most:
            return c


def _sizes(case):
    """Rows and tokens of every sequence: a rule, so that work() knows them too."""
    n, r = case["seqs"], case["rows"]
    if not case["ragged"]:
        rows = [r] * n
    else:
        rows = [0 if s == 2 else max(1, r - (s * 13 % 7) * r // 8) for s in range(n)]
    if case["op"] == "packed":
        return rows, rows
    total = case["ctx"]
    lens = [total] * n if not case["ragged"] else [max(1, total - (s * 29 % 7) * total // 9) for s in range(n)]
    return rows, [max(a, b) for a, b in zip(lens, rows)]


def _first_key(case, rows, length):
    """The first token that any of a sequence's rows sees."""
    return max(0, (length - rows) // case["frame"] - case["window"]) * case["frame"]


def work(case):
    if case["op"] == "norm":
        n, d = case["rows"], case["width"]
        size = {"fp32": 4, "bf16": 2}
        x, y = size[case["x_type"]], size[case["dtype"]]
        moved = n * d * (x + y) if case["first"] else n * d * (2 * x + 2 * y)
        return {"bytes": moved + 3 * case["frames"] * d * 4, "flops": n * d * (18 if case["post"] else 12)}
    size = 4 if case["dtype"] == "fp32" else 2
    h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "rotate":
        return {"bytes": case["rows"] * ((h + hk) * dh * 2 * size + 12), "flops": 3 * case["rows"] * (h + hk) * dh}
    rows, lens = _sizes(case)
    keys = pairs = 0
    f, w = case["frame"], case["window"]
    for r, l in zip(rows, lens):
        keys += l - _first_key(case, r, l) if r else 0
        p = l - r
        if f == 1:                                                         # a causal mask over w + 1 tokens: a sum in closed form
            full = min(r, max(0, l - max(p, w)))                           # rows that see w + 1 tokens
            pairs += full * (w + 1) + sum((p + 1, l - full)) * (r - full) // 2
            continue
        while p < l:                                                       # the rows of one frame see the same keys
            stop = min(l, (p // f + 1) * f)
            pairs += (stop - p) * (stop - max(0, p // f - w) * f)
            p = stop
    n = sum(rows)
    return {"bytes": size * (2 * keys * hk * dh + 2 * n * h * dh), "flops": 4 * pairs * h * dh}


def _cost(case):
    w = work(case)
    most = max(w["bytes"], w["flops"] / 50)
    if case["op"] in ("pages", "packed"):
        rows, lens = _sizes(case)
        span = max(l - _first_key(case, r, l) for r, l in zip(rows, lens))
        most = max(most, case["seqs"] * case["heads"] * max(rows) * span * 5)      # the plain form's scores
        if case["dtype"] == "fp32":
            most = max(most, w["flops"] / 2)
    return most


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
    first = [_first_key(case, r, l) for r, l in zip(rows, lens)]
    return dict(n_rows=n, max_rows=most, row_start=row_start, kv_len=torch.tensor(lens, device=DEV, dtype=torch.int32),
                valid=i[None] < count[:, None], index=row_start[:-1, None].long() + i[None],
                position=(torch.tensor(lens, device=DEV) - count)[:, None] + i[None],
                first=torch.tensor(first, device=DEV), span=max(l - f for l, f in zip(lens, first)))


def _positions(case, gen):
    """Time, row and column [rows, 3] of a video's tokens, the video beginning at a time of its own (frame 1: of a text's)."""
    p = torch.arange(case["rows"], device=DEV)
    f, gw = case["frame"], case["grid_w"]
    t0 = torch.randint(0, 4000, (1,), generator=gen, device=DEV)
    return torch.stack([t0 + p // f, p % f // gw, p % f % gw], 1).int()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(case=case)
    dtype = TYPES[case["dtype"]]
    if case["op"] == "norm":
        n, d, m = case["rows"], case["width"], case["frames"]
        s["x"] = (3 * _randn(gen, n, d) + 0.5).to(TYPES[case["x_type"]])
        s["y"] = None if case["first"] else _randn(gen, n, d, dtype=dtype)
        mod = 0.5 * _randn(gen, m, 3 * d)                       # the modulation's projection: its parts are taken as they lie
        s["gate"], s["scale"], s["shift"] = mod.split(d, dim=1)
        s["index"] = (torch.arange(n, device=DEV) * m // n).int()
        s["weight"] = 1 + 0.1 * _randn(gen, d) if case["post"] else None
        s["x_out"] = None if case["first"] else torch.zeros_like(s["x"])
        s["h"] = torch.zeros(n, d, device=DEV, dtype=dtype)
    else:
        h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
        if case["op"] != "rotate":
            s.update(_rows(case))
        n = case["rows"] if case["op"] == "rotate" else s["n_rows"]
        if case["op"] == "pages":
            s["q"] = _randn(gen, n, h, dh, dtype=dtype)
            p = case["page"]
            per = -(-int(max(_sizes(case)[1])) // p)            # pages that lie in no order, and their table
            s["table"] = torch.randperm(case["seqs"] * per, generator=gen, device=DEV).view(case["seqs"], per).int()
            s["k"] = _randn(gen, case["seqs"] * per, hk, p, dh, dtype=dtype)
            s["k"] *= (1 + 3 * (torch.arange(dh, device=DEV) % 16 == 5)).to(dtype)      # keys have channels that are larger
            s["v"] = _randn(gen, case["seqs"] * per, hk, p, dh, dtype=dtype)
        else:
            qkv = _randn(gen, n, (h + 2 * hk) * dh, dtype=dtype)                         # the projection's output, as it lies
            s["qkv"] = qkv
            s["q"], s["k"], s["v"] = (t.unflatten(1, (-1, dh)) for t in qkv.split([h * dh, hk * dh, hk * dh], dim=1))
        if case["op"] == "rotate":
            s["rope"] = ROPE3[dh] if case["frame"] > 1 else (dh, 0, 0)
            s["pos"] = _positions(case, gen)
            if case["in_place"]:
                s["q_out"], s["k_out"] = s["q"], s["k"]
            else:
                s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        else:
            s["out"] = torch.zeros(n, h * dh, device=DEV, dtype=dtype)
    if own:
        from paper_2506_01380_b200 import nfd as N
        if case["op"] == "norm":
            s["mod"] = N.Modulation(gate=None if case["first"] else s["gate"], scale=s["scale"], shift=s["shift"], index=s["index"])
            s["pre"] = N.Norm(case["kind"], EPS)
            s["post"] = N.Norm(case["kind"], EPS, weight=s["weight"]) if case["post"] and not case["first"] else None
        elif case["op"] == "rotate":
            s["rotation"] = N.Rope(*s["rope"], theta=THETA)
        else:
            s["batch"] = N.Batch(n, s["kv_len"], table=s.get("table"), row_start=s["row_start"], max_rows=s["max_rows"])
            if case["op"] == "pages":
                s["pages"] = N.Pages(s["k"], s["v"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _attention(s, q, k, v, pos):
    """q [B, R, H, dh], k and v [B, L, Hk, dh] fp32 of tokens pos [B, L]; the rows' results go where they belong."""
    case = s["case"]
    b, r, h, dh = q.shape
    hk = k.shape[2]
    frame = s["position"] // case["frame"]                                                    # [B, R]
    lo = (frame - case["window"]).clamp(min=0) * case["frame"]
    hi = torch.minimum((frame + 1) * case["frame"], s["kv_len"][:, None])
    hidden = (pos[:, None] < lo[..., None]) | (pos[:, None] >= hi[..., None])
    v = v.masked_fill((pos >= s["kv_len"][:, None])[..., None, None], 0.0)
    q = q.view(b, r, hk, h // hk, dh).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, dh)          # [B, Hk, heads of the pair x R, dh]
    x = torch.matmul(q, k.permute(0, 2, 3, 1)).mul_(1 / math.sqrt(dh))
    x = x.view(b, h, r, -1).masked_fill_(hidden[:, None], float("-inf"))
    m = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(m == float("-inf"), 0.0, m)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hk, -1, p.shape[-1]), v.transpose(1, 2)).view(b, h, r, dh)
    o = o / torch.where(total == 0, 1.0, total)
    out = torch.zeros_like(s["out"])
    out[s["index"][s["valid"]]] = o.transpose(1, 2)[s["valid"]].flatten(1).to(out.dtype)
    return out


def _padded(s, x):
    return x[s["index"].clamp(max=s["n_rows"] - 1)].float()


def _run_pages(s):
    case = s["case"]
    pos = s["first"][:, None] + torch.arange(s["span"], device=DEV)[None]                    # [B, L]
    page = s["table"].gather(1, (pos // case["page"]).clamp(max=s["table"].shape[1] - 1)).long()
    off = pos % case["page"]
    return _attention(s, _padded(s, s["q"]), s["k"][page, :, off].float(), s["v"][page, :, off].float(), pos)


def _run_packed(s):
    pos = torch.arange(s["max_rows"], device=DEV)[None].expand(s["case"]["seqs"], -1)
    return _attention(s, _padded(s, s["q"]), _padded(s, s["k"]), _padded(s, s["v"]), pos)


def _angles(rope, pos):
    """cos and sin [rows, 1, pairs], fp32, of every pair: the position on its axis times its frequency, in 64 bits."""
    d = torch.tensor(rope, device=DEV)
    pair = torch.arange(sum(rope) // 2, device=DEV)
    axis = (pair >= d[0] // 2).long() + (pair >= (d[0] + d[1]) // 2).long()
    first = torch.stack([d[0] * 0, d[0], d[0] + d[1]])[axis] // 2
    freq = THETA ** (-2.0 * (pair - first).double() / d[axis])
    a = pos.long()[:, axis].double() * freq
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _turn(x, cos, sin, halves):
    x = x.float()
    if halves:
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _run_rotate(s):
    cos, sin = _angles(s["rope"], s["pos"])
    s["q_out"].copy_(_turn(s["q"], cos, sin, s["case"]["halves"]))
    s["k_out"].copy_(_turn(s["k"], cos, sin, s["case"]["halves"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _normed(x, kind):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)


def _run_norm(s):
    case, at = s["case"], s["index"].long()
    x = s["x"].float()
    if not case["first"]:
        t = s["y"].float()
        if case["post"]:
            t = _normed(t, case["kind"]) * s["weight"]
        x = x + 0.5 * s["gate"][at] * t
        s["x_out"].copy_(x)
    s["h"].copy_(_normed(x, case["kind"]) * (1 + s["scale"][at]) + s["shift"][at])
    return {"h": s["h"]} if case["first"] else {"x": s["x_out"], "h": s["h"]}


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        return {"pages": _run_pages, "packed": _run_packed, "rotate": _run_rotate, "norm": _run_norm}[op](s)
    from paper_2506_01380_b200 import nfd as N
    if op == "pages":
        return N.attention_pages(s["pages"], s["batch"], s["q"], s["out"], frame_tokens=case["frame"], window=case["window"])
    if op == "packed":
        return N.attention_packed(s["batch"], s["q"], s["k"], s["v"], s["out"], frame_tokens=case["frame"], window=case["window"])
    if op == "rotate":
        N.rotate(s["rotation"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"], halves=case["halves"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["first"]:
        N.gate_norm(s["x"], h=s["h"], pre=s["pre"], mod=s["mod"])
        return {"h": s["h"]}
    N.gate_norm(s["x"], s["y"], s["x_out"], s["h"], pre=s["pre"], post=s["post"], mod=s["mod"], res_scale=0.5)
    return {"x": s["x_out"], "h": s["h"]}


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, a sequence at a time
# ---------------------------------------------------------------------------------------------------------------
def _turned64(x, rope, pos, halves):
    x = x.double()
    angle = torch.stack([pos[:, a].double() * THETA ** (-2.0 * i / d) for a, d in enumerate(rope) for i in range(d // 2)], 1)[:, None]
    pairs = x.unflatten(-1, (2, -1)).transpose(-1, -2) if halves else x.unflatten(-1, (-1, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.polar(torch.ones_like(angle), angle))
    return (z.transpose(-1, -2) if halves else z).flatten(-2)


def _normed64(x, kind):
    var, mean = torch.var_mean(x, -1, keepdim=True, correction=0)
    if kind == "rms":
        var, mean = var + mean ** 2, torch.zeros_like(mean)
    return (x - mean) * torch.rsqrt(var + EPS)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        row = lambda t: torch.repeat_interleave(t.double(), torch.bincount(s["index"], minlength=case["frames"]), dim=0)
        x = s["x"].double()
        if not case["first"]:
            t = _normed64(s["y"].double(), case["kind"]) * s["weight"].double() if case["post"] else s["y"].double()
            x = x + row(s["gate"]) * t / 2
        h = torch.addcmul(row(s["shift"]), _normed64(x, case["kind"]), row(s["scale"]) + 1)
        return {"h": h} if case["first"] else {"x": x, "h": h}
    if case["op"] == "rotate":
        return {n: _turned64(s[n], s["rope"], s["pos"], case["halves"]) for n in ("q", "k")}
    rows, lens = _sizes(case)
    h, hk, dh = case["heads"], case["kv_heads"], case["head_dim"]
    start = s["row_start"].tolist()
    out = torch.zeros(s["n_rows"], h, dh, device=DEV, dtype=torch.float64)
    for b, (r, l) in enumerate(zip(rows, lens)):
        if not r:
            continue
        here = slice(start[b], start[b] + r)
        pos = torch.arange(_first_key(case, r, l), l, device=DEV)
        if case["op"] == "pages":
            page, off = s["table"][b].long()[pos // case["page"]], pos % case["page"]
            k, v = s["k"][page, :, off].double(), s["v"][page, :, off].double()
        else:
            k, v = s["k"][here].double(), s["v"][here].double()
        fq, fk = torch.arange(l - r, l, device=DEV) // case["frame"], pos // case["frame"]
        hidden = (fk[None] > fq[:, None]) | (fk[None] < fq[:, None] - case["window"])
        for head in range(h):
            g = head * hk // h
            x = s["q"][here, head].double() @ k[:, g].T / math.sqrt(dh)
            x.masked_fill_(hidden, float("-inf"))
            out[here, head] = torch.softmax(x, 1) @ v[:, g]
    return out.flatten(1)
