"""The calls around a block's projections against the 64-bit oracle: attention over bf16 and fp32 pages, attention over packed
prompts, rotation, norms with gate and residual, and a run of them together.

Bounds of attention.  With S = |q||k| / sqrt(dh), a score is off by at most (dh + 2) 2^-23 S in its fp32 sum (tensor cores may
truncate where they add), its exponential by that, S 2^-23 (argument) and 2^-21 (function): together e.  A result o = sum p v / sum p
is off by 2 e M (numerator and denominator), M = sum p |v| / sum p, n 2^-23 M for its sums over n keys and the rounding of
itself: 2^-23 |o| in fp32, 2^-8 |o| in bf16, where probabilities rounded to bf16 add 2^-8 M.  (1 % on these two is for the
products of roundings.)
Bounds of a rotation.  The angle is off by 2^-24 turns in fp32 (2 pi 2^-24 < 2^-21) and the 64-bit product by |position| 2^-52;
sine and cosine by that and 2^-22; u = a c - b s by that times |a| + |b|, three roundings of 2^-24 (|a| + |b|) and its own, 2^-24 |u| or 2^-9 |u|.
Bounds of a norm.  Sums of n terms are off by n 2^-24 relative to the sum of their magnitudes at the very most; here a thread adds up to
32 in a row and the rest is a tree of at most 10 levels: 48 2^-24.  See _check_norm.
"""
import numpy as np
import pytest

from oracle import block_oracle as O

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
EVER = (1 << 31) - 1


def _mods():
    import torch
    from paper_2506_01380_b200 import nfd as N
    return torch, N


def _int(a):
    torch, _ = _mods()
    return torch.as_tensor(np.asarray(a, np.int32)).cuda()


def _batch(rows, lens=None, table=None, extra=0, max_rows=None):
    """(Batch, n_rows, first row of each) of sequences with `rows` rows and `lens` tokens; `extra` rows behind the last one."""
    torch, N = _mods()
    start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    n = int(start[-1]) + extra
    b = N.Batch(n, _int(lens) if lens is not None else None, table=table, row_start=_int(start), n_seqs=len(rows),
                max_rows=max_rows if max_rows is not None else max(list(rows) + [0]))
    return b, n, start


def _within(got, want, mag, smax, n, dh, half):
    torch, _ = _mods()
    e = (dh + 4) * 2.0 ** -23 * smax + 2.0 ** -21
    own = 1.01 * half if half else 2.0 ** -23
    bound = (2 * e + n * 2.0 ** -23 + 1.01 * half) * mag + own * want.abs() + 1e-30
    nan = want.isnan()
    off = torch.where(nan, 0.0, (got.double() - want).abs() - bound)
    assert torch.isfinite(got[~nan]).all() and not torch.isfinite(got[nan]).any()
    assert (off <= 0).all(), (off.max().item(), (got.double() - want).abs().nan_to_num().max().item())


def _smax(q, k):
    norm = lambda x: x.double().nan_to_num(0, 0, 0).norm(dim=-1).max().item() if x.numel() else 0.0
    return norm(q) * norm(k) / np.sqrt(q.shape[-1])


def _randn(g, *shape, dtype):
    torch, _ = _mods()
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _check_pages(dtype, rows, lens, heads, share, dh, page, table_len, frame, window, seed=0, extra=0, scale=1.0, table=None, n_pages=None,
                 poke=None, max_rows=None, pad=0):
    """Pages in no order, some beyond any table; a ring where table_len pages do not hold a sequence."""
    torch, N = _mods()
    g = torch.Generator("cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt, hk, S = getattr(torch, dtype), heads // share, len(rows)
    if table is None:
        n_pages = S * table_len + 3
        table = rng.permutation(n_pages)[:S * table_len].reshape(S, table_len).astype(np.int32)
    k, v = (_randn(g, n_pages, hk, page, dh, dtype=dt) for _ in range(2))
    if poke is not None:
        poke(k, v, table)
    b, n, start = _batch(rows, lens, _int(table), extra, max_rows)
    q = (_randn(g, n, heads * dh + pad, dtype=torch.float32) * scale).to(dt)[:, :heads * dh].unflatten(1, (heads, dh))
    out = torch.full((n, heads * dh), 7.0, device="cuda", dtype=dt)
    N.attention_pages(N.Pages(k, v), b, q, out, frame_tokens=frame, window=window)
    got = out.view(n, heads, dh)
    live = torch.zeros(n, dtype=torch.bool)
    for s, (r, length) in enumerate(zip(rows, lens)):
        t = np.arange(length)
        pg = table[s][(t // page) % table.shape[1]]
        held = (t >= length - table.shape[1] * page) & (pg >= 0) & (pg < n_pages)
        seen = O.seen_tokens(r, length, frame, window)[:, held]
        pg, off = torch.as_tensor(pg[held]).long().cuda(), torch.as_tensor((t % page)[held]).cuda()
        kk, vv = k[pg, :, off], v[pg, :, off]
        here = slice(start[s], start[s] + r)
        want, mag = O.attend(q[here], kk, vv, seen)
        cap = r if max_rows is None else min(r, max_rows)
        live[start[s]:start[s] + cap] = True
        _within(got[here][:cap], want[:cap], mag[:cap], _smax(q[here], kk), length, dh, HALF if dtype == "bfloat16" else 0.0)
    assert (got[~live.cuda()] == 7).all()
    return got


def _check_packed(dtype, rows, heads, share, dh, frame, window, seed=0, extra=0, scale=1.0, poke=None, max_rows=None, fused=True, uniform=False):
    torch, N = _mods()
    g = torch.Generator("cuda").manual_seed(seed)
    dt, hk = getattr(torch, dtype), heads // share
    b, n, start = _batch(rows, None, None, extra, max_rows)
    if uniform:
        b = N.Batch(n, n_seqs=len(rows))
    x = (_randn(g, n, (heads + 2 * hk) * dh, dtype=torch.float32) * scale).to(dt)
    q, k, v = (t.unflatten(1, (-1, dh)) for t in x.split([heads * dh, hk * dh, hk * dh], 1))
    if not fused:
        q, k, v = (t.contiguous() for t in (q, k, v))
    if poke is not None:
        poke(q, k, v)
    out = torch.full((n, heads * dh), 7.0, device="cuda", dtype=dt)
    N.attention_packed(b, q, k, v, out, frame_tokens=frame, window=window)
    got = out.view(n, heads, dh)
    live = torch.zeros(n, dtype=torch.bool)
    for s, r in enumerate(rows):
        here, cap = slice(start[s], start[s] + r), r if max_rows is None else min(r, max_rows)
        want, mag = O.attend(q[here], k[here], v[here], O.seen_tokens(r, r, frame, window))
        live[start[s]:start[s] + cap] = True
        _within(got[here][:cap], want[:cap], mag[:cap], _smax(q[here], k[here]), r, dh, HALF if dtype == "bfloat16" else 0.0)
    assert (got[~live.cuda()] == 7).all()
    return got


TYPES = ["bfloat16", "float32"]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("heads,share,rows,lens,page,table_len,frame,window", [
    (4, 1, [1, 1, 1], [1, 77, 300], 16, 20, 1, EVER),                  # single tokens, the first of all among them
    (6, 3, [1, 4, 0, 2], [300, 40, 7, 2], 11, 30, 1, 50),              # a window, a sequence without rows
    (2, 1, [130, 40], [220, 61], 64, 4, 1, EVER),                      # a chunk across tiles, a ragged one
    (4, 4, [33, 7, 100], [228, 7, 129], 7, 33, 5, 3),                  # frames, heads that share, small pages
    (3, 1, [257], [257], 300, 1, 64, 1)])                              # from the start on, the page larger than the sequence
def test_pages(dtype, dh, heads, share, rows, lens, page, table_len, frame, window):
    _check_pages(dtype, rows, lens, heads, share, dh, page, table_len, frame, window, seed=dh, extra=2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 3, 8, 17, 60, 64, 65, 127, 128, 129, 256, 257, 300])
def test_pages_rows_and_keys_around_the_tiles(dtype, rows):
    for keys in (0, 1, 31, 95, 96, 97, 128, 500):
        _check_pages(dtype, [rows], [rows + keys], 2, 1, 64, 50, 17, 1, EVER, seed=rows + keys)
        _check_pages(dtype, [rows], [rows + keys], 2, 2, 128, 64, 13, 1, EVER, seed=rows + keys)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("rows,length,heads,share", [(336, 2000, 16, 1), (100, 5712, 2, 1), (700, 3000, 8, 4), (1000, 1000, 1, 1), (90, 9000, 1, 1)])
def test_pages_split_and_whole(dh, rows, length, heads, share):
    """One tile and two to a CTA, keys split over clusters and not."""
    _check_pages("bfloat16", [rows], [length], heads, share, dh, 64, length // 64 + 1, 1, EVER, seed=rows)
    _check_pages("bfloat16", [rows] * 7, [length] * 7, heads, share, dh, 64, length // 64 + 1, 1, EVER, seed=rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [2, 150, 400])
def test_pages_windows(dtype, rows):
    for frame, window in ((1, 0), (1, 1), (1, 100), (7, 0), (7, 2), (336, 1), (1000, 0), (1, 300)):
        _check_pages(dtype, [rows, rows // 2], [900, 640], 4, 2, 64, 48, 19, frame, window, seed=rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 150, 300])
def test_pages_rows_that_see_nothing(dtype, rows):
    """No tokens at all, tokens below 0, every page missing: zeros; a hole in the table: its keys are seen by nobody; a ring."""
    gone = np.full((3, 12), -1, np.int32)
    assert (_check_pages(dtype, [rows] * 3, [0, 180, 180], 2, 1, 64, 16, 12, 1, EVER, table=gone, n_pages=12) == 0).all()
    rng = np.random.default_rng(0)
    holes = np.array([rng.permutation(12) for _ in range(3)], np.int32)
    holes[0, 3:6], holes[1, 0], holes[2, 11] = -7, 12, 1 << 30
    _check_pages(dtype, [rows] * 3, [180, 170, 192], 2, 1, 64, 16, 12, 1, EVER, table=holes, n_pages=12)
    got = _check_pages(dtype, [rows], [rows // 2], 2, 1, 64, 16, 12, 1, EVER, table=holes[:1], n_pages=12)
    assert (got[:rows - rows // 2] == 0).all()
    _check_pages(dtype, [rows, rows], [1000, 333], 2, 1, 64, 16, 12, 1, EVER, extra=1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("rows,share", [(3, 1), (3, 4), (20, 1), (150, 1), (300, 2)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_pages_values_that_are_not_finite(dtype, dh, rows, share, value):
    """In a value: its column of the rows that see it, and nothing else.  Where nobody looks (keys and values behind the end, in
    front of the window): nothing."""
    length, window = 500, 200

    def poke(k, v, table):
        for t in list(range(0, length - rows - window)) + list(range(length, 520)):
            k[table[0][t // 40], :, t % 40] = v[table[0][t // 40], :, t % 40] = value
        for t, d in ((length - 1, 3), (length - rows // 2 - 1, 17), (length - rows - window + rows // 3, dh - 1)):
            v[table[0][t // 40], 0, t % 40, d] = value
    _check_pages(dtype, [rows], [length], 2 * share, share, dh, 40, 13, 1, window, seed=3, poke=poke)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_pages_scores_flat_peaked_and_rising(dtype, rows):
    """Equal scores; scores far apart; the largest last, far above the first ones; the type's lowest value among the keys."""
    for scale in (0.0, 30.0):
        _check_pages(dtype, [rows], [900], 2, 1, 64, 100, 9, 1, EVER, scale=scale)

    def rising(k, v, table):
        k[..., 0] = 0
        for t in range(900):
            k[table[0][t // 100], :, t % 100, 0] = t / 3.0
    for dh in (64, 128):
        _check_pages(dtype, [rows], [900], 2, 1, dh, 100, 9, 1, EVER, scale=8.0, poke=rising)

    def lowest(k, v, table):
        import torch
        k[table[0][2], :, 5] = torch.finfo(k.dtype).min / 4096
    _check_lowest(dtype, rows, lowest)


def _check_lowest(dtype, rows, poke):
    """Keys of the lowest values there are: scores of +-10^34 or so, finite in fp32; the rest must not suffer."""
    torch, N = _mods()
    g = torch.Generator("cuda").manual_seed(1)
    dt = getattr(torch, dtype)
    k, v = (_randn(g, 9, 2, 100, 64, dtype=dt) for _ in range(2))
    table = np.arange(9, dtype=np.int32)[None]
    poke(k, v, table)
    b, n, _ = _batch([rows], [900], _int(table))
    q = _randn(g, n, 2, 64, dtype=dt).abs()                            # (so that these scores are the lowest)
    out = torch.zeros(n, 128, device="cuda", dtype=dt)
    N.attention_pages(N.Pages(k, v), b, q, out)
    seen = O.seen_tokens(rows, 900, 1, EVER)
    seen[:, 205] = False                                               # their probability is 0
    kk, vv = (t.transpose(1, 2).flatten(0, 1) for t in (k, v))
    want, mag = O.attend(q, kk, vv, seen)
    ok = torch.ones(900, dtype=torch.bool)
    ok[205] = False
    _within(out.view(n, 2, 64), want, mag, _smax(q, kk[ok.cuda()]), 900, 64, HALF if dtype == "bfloat16" else 0.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 40, 300])
def test_values_as_large_as_the_type_goes(dtype, rows):
    import torch

    def poke(k, v, table):
        v.copy_(torch.where(v > 0, 1.0, -1.0).to(v.dtype) * torch.finfo(v.dtype).max * 0.99)
    torch_, N = _mods()
    g = torch.Generator("cuda").manual_seed(2)
    dt = getattr(torch, dtype)
    k, v = (_randn(g, 40, 1, 64, 64, dtype=dt) for _ in range(2))
    poke(k, v, None)
    v[:, :, :, 0] = v[:, :, :, 0].abs()                                # a column whose mean is the largest value
    b, n, _ = _batch([rows], [40 * 64], _int(np.arange(40)[None]))
    q = _randn(g, n, 1, 64, dtype=dt) * 4
    out = torch.zeros(n, 64, device="cuda", dtype=dt)
    N.attention_pages(N.Pages(k, v), b, q, out)
    want, mag = O.attend(q, k.flatten(0, 2)[:, None], v.flatten(0, 2)[:, None], O.seen_tokens(rows, 40 * 64, 1, EVER))
    s = 2.0 ** -100
    _within(out.double().view(n, 1, 64) * s, want * s, mag * s, _smax(q, k), 2560, 64, HALF if dtype == "bfloat16" else 0.0)


def test_pages_offsets_beyond_32_bits():
    """A cache of more than 2^32 numbers, with the sequence's pages at its end."""
    torch, N = _mods()
    page, dh = 512, 128
    n_pages = (1 << 32) // (page * 8 * dh) + 32
    k, v = (torch.zeros(n_pages, 8, page, dh, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.arange(n_pages - 3, n_pages, device="cuda", dtype=torch.int32).flip(0)[None].contiguous()
    k[-3:], v[-3:] = torch.randn_like(k[-3:]), torch.randn_like(v[-3:])
    kv = _int([1500])
    for n in (1, 40, 300):
        q = torch.randn(n, 8, dh, device="cuda").bfloat16()
        o1, o2 = (torch.zeros(n, 8 * dh, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        N.attention_pages(N.Pages(k, v), N.Batch(n, kv, table), q, o1)
        N.attention_pages(N.Pages(k[-3:].clone(), v[-3:].clone()), N.Batch(n, kv, _int([[2, 1, 0]])), q, o2)
        assert torch.equal(o1, o2) and o1.abs().sum() > 0


def test_pages_capped_rows_and_strides():
    for rows, cap in (([20, 9], 13), ([300, 200], 260)):
        _check_pages("bfloat16", rows, [400, 350], 4, 2, 64, 16, 25, 1, EVER, max_rows=cap, extra=1, pad=64)
        _check_pages("float32", rows, [400, 350], 4, 2, 64, 16, 25, 1, EVER, max_rows=cap, extra=1, pad=64)


# ---------------------------------------------------------------------------------------------------------------
# packed prompts
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("heads,share,rows,frame,window", [
    (4, 1, [1, 1, 1], 1, EVER),
    (6, 3, [5, 0, 60, 1], 1, EVER),
    (2, 1, [130, 257, 1, 40], 1, EVER),
    (8, 4, [33, 300, 100], 1, 70),
    (4, 2, [220, 77, 231], 77, 1),
    (2, 2, [400, 200], 500, 0)])                                       # a frame longer than the sequence: all of it
def test_packed(dtype, dh, heads, share, rows, frame, window):
    _check_packed(dtype, rows, heads, share, dh, frame, window, seed=dh, extra=3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 8, 31, 63, 64, 65, 95, 96, 97, 127, 128, 129, 191, 192, 193, 255, 256, 257, 383, 384, 385, 513])
def test_packed_lengths_around_the_tiles(dtype, rows):
    for dh in (64, 128):
        _check_packed(dtype, [rows], 2, 1, dh, 1, EVER, seed=rows)
        _check_packed(dtype, [rows, rows], 2, 2, dh, 1, 90, seed=rows, uniform=True, fused=False)


@pytest.mark.parametrize("dh", [64, 128])
def test_packed_long(dh):
    _check_packed("bfloat16", [3000, 77, 1500], 8, 4, dh, 1, EVER)
    _check_packed("bfloat16", [2100], 1, 1, dh, 1, EVER)
    _check_packed("bfloat16", [16 * 77] * 3, 4, 1, dh, 77, 3)


@pytest.mark.parametrize("n_seqs", [33, 128, 129, 300])
def test_packed_many_sequences(n_seqs):
    rng = np.random.default_rng(n_seqs)
    rows = [int(r) for r in rng.integers(0, 400, n_seqs)]
    _check_packed("bfloat16", rows, 2, 1, 64, 1, EVER, extra=5)
    _check_packed("bfloat16", [r // 10 for r in rows], 2, 1, 64, 1, EVER, extra=5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [3, 40, 150, 300, 700])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_packed_values_that_are_not_finite(dtype, rows, value):
    """In a value: its column of the rows from there on.  In the rows of a neighbour, behind the last sequence: nothing."""
    def poke(q, k, v):
        q[-2:] = k[-2:] = v[-2:] = value
        for t, d in ((rows - 1, 3), (rows - rows // 3, 17), (rows // 2, 31)):
            v[t, 0, d] = value
        k[rows + 5:rows + 10] = value                                  # the next sequence's rows from there on are not finite
    import torch
    torch_, N = _mods()
    for dh in (64, 128):
        g = torch.Generator("cuda").manual_seed(0)
        dt = getattr(torch, dtype)
        b, n, _ = _batch([rows, 20], None, None, 2)
        q, k, v = (_randn(g, n, 2, dh, dtype=dt) for _ in range(3))
        poke(q, k, v)
        out = torch.full((n, 2 * dh), 7.0, device="cuda", dtype=dt)
        N.attention_packed(b, q, k, v, out)
        got = out.view(n, 2, dh)
        want, mag = O.attend(q[:rows], k[:rows], v[:rows], O.seen_tokens(rows, rows, 1, EVER))
        _within(got[:rows], want, mag, _smax(q[:rows], k[:rows]), rows, dh, HALF if dtype == "bfloat16" else 0.0)
        here = slice(rows, rows + 5)
        want, mag = O.attend(q[here], k[here], v[here], O.seen_tokens(5, 5, 1, EVER))
        _within(got[here], want, mag, _smax(q[here], k[here]), 5, dh, HALF if dtype == "bfloat16" else 0.0)
        assert (got[-2:] == 7).all()


def test_packed_capped_rows():
    _check_packed("bfloat16", [300, 200], 2, 1, 64, 90, EVER, max_rows=150)
    _check_packed("float32", [300, 200], 2, 1, 64, 90, EVER, max_rows=150)
    _check_packed("bfloat16", [30, 20], 2, 1, 64, 9, EVER, max_rows=14)


def test_packed_is_pages_of_the_same_rows():
    """The rows of a prompt and the same rows in pages that lie in order: the same numbers to the bit."""
    torch, N = _mods()
    for dh, n in ((64, 700), (128, 700), (64, 30)):
        q, k, v = (torch.randn(n, 4, dh, device="cuda").bfloat16() for _ in range(3))
        o1, o2 = (torch.zeros(n, 4 * dh, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        N.attention_packed(N.Batch(n, row_start=_int([0, n]), max_rows=n), q, k, v, o1, frame_tokens=50, window=5)
        pages = N.Pages(*(t.transpose(0, 1).contiguous()[None] for t in (k, v)))
        N.attention_pages(pages, N.Batch(n, _int([n]), _int([[0]])), q, o2, frame_tokens=50, window=5)
        assert torch.equal(o1, o2)


# ---------------------------------------------------------------------------------------------------------------
# rotation
# ---------------------------------------------------------------------------------------------------------------
def _check_rotate(dtype, n, heads, heads2, dh, rope, halves, back, far=1000, in_place=False, seed=0):
    torch, N = _mods()
    dt = getattr(torch, dtype)
    g = torch.Generator("cuda").manual_seed(seed)
    pos = torch.randint(-far, far, (n, 3), generator=g, device="cuda").int()
    x = _randn(g, n, (heads + heads2) * dh + 16, dtype=dt)
    a, b = x[:, :heads * dh].unflatten(1, (heads, dh)), x[:, heads * dh:(heads + heads2) * dh].unflatten(1, (heads2, dh)) if heads2 else None
    old = x.clone()
    oa = a if in_place else torch.full_like(a, 7.0).contiguous()
    ob = None if b is None else b if in_place else torch.full_like(b, 7.0).contiguous()
    N.rotate(N.Rope(*rope, theta=1e4), pos, a, oa, b, ob, halves=halves, back=back)
    o = old[:, :heads * dh].unflatten(1, (heads, dh)), old[:, heads * dh:(heads + heads2) * dh].unflatten(1, (heads2, dh)) if heads2 else None
    for got, src in ((oa, o[0]), (ob, o[1])):
        if got is None:
            continue
        want = O.rotate(src, pos, rope, 1e4, halves, back)
        s = src.double().abs()
        p, q = s.chunk(2, -1) if halves else (s[..., 0::2], s[..., 1::2])
        both = torch.cat([p + q] * 2, -1) if halves else (p + q).repeat_interleave(2, -1)
        # (either side's 64-bit angle is off by a few ulps of its frequency and product)
        bound = both * (2.0 ** -21 + 2.0 ** -22 + far * 2.0 ** -50 + 3 * 2.0 ** -24) + want.abs() * (2.0 ** -24 if dtype == "float32" else 1.01 * 2.0 ** -8)
        assert ((got.double() - want).abs() <= bound).all(), ((got.double() - want).abs() - bound).max().item()
    if in_place:
        assert torch.equal(x[:, (heads + heads2) * dh:], old[:, (heads + heads2) * dh:])
    else:
        assert torch.equal(x, old)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("dh,rope", [(32, (8, 12, 12)), (64, (16, 24, 24)), (64, (64, 0, 0)), (128, (0, 64, 64)), (16, (2, 6, 8)), (256, (64, 96, 96)), (80, (16, 32, 32))])
def test_rotate(dtype, halves, dh, rope):
    for n, heads, heads2 in ((1, 1, 0), (8, 16, 4), (77, 3, 3), (1300, 5, 1)):
        _check_rotate(dtype, n, heads, heads2, dh, rope, halves, False, seed=n)
        _check_rotate(dtype, n, heads, heads2, dh, rope, halves, True, seed=n, in_place=True)


def test_rotate_far_positions_and_none():
    _check_rotate("float32", 500, 2, 1, 64, (16, 24, 24), False, False, far=(1 << 31) - 1)
    torch, N = _mods()
    empty = torch.zeros(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    N.rotate(N.Rope(64, 0, 0), torch.zeros(0, 3, device="cuda", dtype=torch.int32), empty)


def test_rotate_back_undoes_and_is_the_gradient():
    """Against differences: the derivative of a weighted sum of the rotated numbers in direction e is <weights turned back, e>."""
    torch, N = _mods()
    for halves in (False, True):
        r, pos = N.Rope(16, 24, 24), torch.randint(0, 300, (50, 3), device="cuda").int()
        x, w, e = (torch.randn(50, 3, 64, device="cuda") for _ in range(3))
        turned = lambda t, **kw: N.rotate(r, pos, t, torch.empty_like(t), halves=halves, **kw)[0]
        assert (turned(turned(x), back=True) - x).abs().max() < 2e-6
        along = ((turned(x + e) - turned(x - e)).double() * w.double()).sum() / 2
        assert abs(along - (turned(w, back=True).double() * e.double()).sum()) < 1e-3


def test_rotate_is_what_append_writes():
    """Positions of a grid: the rotation that rows get on their way into a cache, to fp32's last bits."""
    torch, N = _mods()
    n, frame, gw = 400, 77, 7
    k = torch.randn(n, 3, 64, device="cuda")
    pages = N.Pages.empty(torch.float32, 1, 3, n, 64)
    b = N.Batch(n, _int([n]), _int([[0]]))
    N.kv_append(pages, b, k, k, N.Rope(16, 24, 24, frame_tokens=frame, grid_w=gw))
    p = torch.arange(n, device="cuda")
    pos = torch.stack([p // frame, p % frame // gw, p % frame % gw], 1).int()
    N.rotate(N.Rope(16, 24, 24), pos, k)
    assert (k - pages.k[0].transpose(0, 1)).abs().max() <= 2.0 ** -20 * k.abs().max()


# ---------------------------------------------------------------------------------------------------------------
# norms around a block
# ---------------------------------------------------------------------------------------------------------------
def _check_norm(xt, dt, n, width, kind, post, gate, scale, shift, affine, ptype="float32", use_y=True, use_h=True, index=True, seed=0, mean=0.0, in_place=False):
    """Errors, in units u = 2^-24: a sum is off by up to 48 u of its terms' magnitudes, a mean square by that and its terms' own 2 u, its
    root by half of it; with LayerNorm the mean is off by 48 u mean |x|, which is 48 u A, A = rms(x) for short, and by that and u |x| each difference.  So normed(x) is off by
    e = (48 A + |x| + 2 A) u / std + |normed(x)| 32 u (root, quotient, their roundings): then what is done to it, a rounding each."""
    torch, N = _mods()
    g = torch.Generator("cuda").manual_seed(seed)
    tx, ty, tp = (getattr(torch, t) for t in (xt, dt, ptype))
    pad = 24
    wide = lambda rows, t, m=0.0: (_randn(g, rows, width + pad, dtype=torch.float32) * 2 + m).to(t)[:, :width]
    x, y = wide(n, tx, mean), wide(n, ty, mean) if use_y else None
    n_mods = 5
    mods = (_randn(g, n_mods, 3 * width, dtype=torch.float32) * 0.5).to(tp)
    gt, sc, sh = (m if on else None for m, on in zip(mods.split(width, 1), (gate, scale, shift)))
    par = lambda on, m: (m + 0.3 * _randn(g, width, dtype=torch.float32)).to(tp) if on else None
    eps = 1e-5
    po = (kind, eps, par(affine, 1.0), par(affine, 0.0)) if post else None
    pr = (kind, eps, par(affine, 1.0), par(affine, 0.0)) if use_h else None
    which = torch.randint(-2, n_mods + 2, (n,), generator=g, device="cuda").int()
    mod = None
    if gate or scale or shift:
        mod = N.Modulation(gt, sc, sh, index=which) if index else N.Modulation(gt, sc, sh, rows_per_mod=max(1, n // 3))
    at = which.long().clamp(0, n_mods - 1) if index else (torch.arange(n, device="cuda") // max(1, n // 3)).clamp(max=n_mods - 1)
    row = lambda m: m[at] if m is not None else None
    x0 = x.clone()
    y0 = y.clone() if use_y else None
    h = None if not use_h else y if in_place and use_y else torch.full((n, width), 7.0, device="cuda", dtype=ty)
    xo = None if not use_y else x if in_place else torch.full((n, width), 7.0, device="cuda", dtype=tx)
    norm = lambda p: N.Norm(p[0], p[1], p[2], p[3]) if p is not None else None
    N.gate_norm(x, y, xo, h, pre=norm(pr), post=norm(po), mod=mod, res_scale=0.7)
    want_x, want_h = O.gate_norm(x0, y0, po, pr, row(gt), row(sc), row(sh), float(np.float32(0.7)))
    u = 2.0 ** -24
    rms = lambda t: (t * t).mean(-1, keepdim=True).sqrt()
    own = lambda t, w: w.abs() * (u if t == "float32" else 2.0 ** -8)

    def normed_error(t, before, p):
        """of normed(t), whose numbers are off by `before` to begin with"""
        d = t - t.mean(-1, keepdim=True) if kind == "layer" else t
        std = torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
        off = before + (50 * rms(t) + t.abs()) * u if kind == "layer" else before + 0 * t
        z = d / std
        e = (off + rms(off) * z.abs()) / std + z.abs() * 32 * u
        if p[2] is not None:
            e = e * p[2].double().abs() + (z * p[2].double()).abs() * 2 * u
        return e + (3 * u) * O.normed(t, *p).abs() + (2 * u * p[3].double().abs() if p[3] is not None else 0)
    e = 0 * x0.double()
    if use_y:
        t = O.normed(y0, *po) if post else y0.double()
        e = normed_error(y0.double(), e, po) if post else e
        factor = 0.7 * (row(gt).double().abs() if gate else 1.0)
        e = factor * (e + 3 * u * t.abs()) + u * want_x.abs()
        assert ((xo.double() - want_x).abs() <= 1.01 * (e + own(xt, want_x)) + 1e-30).all()
    elif not in_place:
        assert torch.equal(x, x0)
    if use_h:
        z = O.normed(want_x, *pr)
        e = normed_error(want_x, e, pr)
        if scale:
            e = e * (1 + row(sc).double().abs()) + 2 * u * z.abs() * (1 + row(sc).double().abs())
        e = e + 2 * u * want_h.abs() + (u * row(sh).double().abs() if shift else 0)
        off = (h.double() - want_h).abs() - 1.01 * (e + own(dt, want_h)) - 1e-30
        assert (off <= 0).all(), off.max().item()


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("xt,dt,ptype", [("float32", "bfloat16", "float32"), ("float32", "float32", "bfloat16"), ("bfloat16", "bfloat16", "bfloat16"),
                                         ("bfloat16", "float32", "float32")])
def test_gate_norm(kind, xt, dt, ptype):
    for n, width in ((1, 8), (5, 64), (336, 1024), (37, 1032), (3, 2056), (2, 8200), (2, 16384), (2500, 264), (2500, 520), (2400, 1024)):
        _check_norm(xt, dt, n, width, kind, True, True, True, True, True, ptype, seed=width)
        _check_norm(xt, dt, n, width, kind, False, True, True, True, False, ptype, seed=width, in_place=True)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate,scale,shift", [(0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1)])
def test_gate_norm_parts(post, gate, scale, shift):
    for use_y, use_h in ((True, True), (True, False), (False, True)):
        for index in (False, True):
            _check_norm("float32", "bfloat16", 40, 520, "layer", post and use_y, gate, scale, shift, post, use_y=use_y, use_h=use_h, index=index)


def test_gate_norm_far_from_zero():
    """A mean a thousand times the deviation: the squares are taken of what is left when it is gone."""
    for width in (512, 1024, 4096):
        _check_norm("float32", "float32", 30, width, "layer", False, True, True, True, True, mean=2000.0)


def test_gate_norm_not_finite():
    """A row with a NaN or an infinity in it is its own affair."""
    torch, N = _mods()
    for width in (256, 1024, 4096):
        x, y = torch.randn(9, width, device="cuda"), torch.randn(9, width, device="cuda").bfloat16()
        run = lambda: N.gate_norm(x, y, torch.empty_like(x), torch.empty_like(y), pre=N.Norm("layer"), post=N.Norm("rms"))
        a = run()
        x[3, 5], y[6, 7] = float("nan"), float("inf")
        b = run()
        keep = [0, 1, 2, 4, 5, 7, 8]
        assert all(torch.equal(p[keep], q[keep]) for p, q in zip(a, b)) and b[1][3].isnan().all() and b[1][6].isnan().all()


# ---------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------
def _block64(x, w, mod, kind, rope, pos, spans, heads, share, dh, frame, window):
    """A pre-norm block in 64 bits: norm, projection, rotation, attention per span, projection, gate."""
    import torch
    hk = heads // share
    _, h = O.gate_norm(x, None, None, (kind, 1e-6, None, None), None, mod[1], mod[2], 1.0)
    q, k, v = (t.unflatten(1, (-1, dh)) for t in (h @ w[0].double()).split([heads * dh, hk * dh, hk * dh], 1))
    q, k = O.rotate(q, pos, rope, 1e4), O.rotate(k, pos, rope, 1e4)
    o = torch.cat([O.attend(q[a:b], k[a:b], v[a:b], O.seen_tokens(b - a, b - a, frame, window))[0] for a, b in spans]).flatten(1)
    return O.gate_norm(x, o @ w[1].double(), (kind, 1e-6, None, None), (kind, 1e-6, None, None), mod[0], mod[1], mod[2], 1.0)


def test_block_prompt_then_frames():
    """A block as a host runs it: two prompts in one packed pass, rows into pages, then a frame more over the pages, with replays of a
    captured graph: what comes out is what the 64-bit block says of the whole sequence."""
    torch, N = _mods()
    heads, share, dh, frame, gw, window, width = 8, 2, 64, 48, 8, 3, 256
    hk, rope = heads // share, (16, 24, 24)
    g = torch.Generator("cuda").manual_seed(0)
    w = ((_randn(g, width, (heads + 2 * hk) * dh, dtype=torch.float32) / 16).bfloat16(), (_randn(g, heads * dh, width, dtype=torch.float32) / 22).bfloat16())
    frames = (4, 6)                                                    # of the two prompts; then one frame more each
    total = [(f + 1) * frame for f in frames]
    xs = [_randn(g, t, width, dtype=torch.float32) for t in total]
    mods = _randn(g, 1, 3 * width, dtype=torch.float32) * 0.3
    mod = N.Modulation(*mods.split(width, 1), rows_per_mod=1 << 20)
    pre, post, R = N.Norm("rms"), N.Norm("rms"), N.Rope(*rope, frame_tokens=frame, grid_w=gw)
    pages = N.Pages.empty(torch.bfloat16, 40, hk, 20, dh)
    table = torch.randperm(40, generator=g, device="cuda")[:2 * 18].view(2, 18).int()
    kv_len = _int([f * frame for f in frames])

    def step(x, spans_rows, pos, packed):
        n = x.shape[0]
        new = lambda *sh, dt=torch.bfloat16: torch.zeros(sh, device="cuda", dtype=dt)
        start = _int(np.concatenate([[0], np.cumsum(spans_rows)]))
        b = N.Batch(n, kv_len, table=table, row_start=start, max_rows=max(spans_rows))
        h, qr, out = new(n, width), new(n, heads, dh), new(n, heads * dh)
        x_out, h_out = new(n, width, dt=torch.float32), new(n, width)

        def run():
            N.gate_norm(x, h=h, pre=pre, mod=mod)
            q, k, v = (t.unflatten(1, (-1, dh)) for t in (h @ w[0]).split([heads * dh, hk * dh, hk * dh], 1))
            if packed:
                N.kv_append(pages, b, k, v, R)
                N.rotate(R, pos, q, x2=k)
                N.attention_packed(b, q, k, v, out, frame_tokens=frame, window=window)
            else:
                N.kv_append(pages, b, k, v, R, q=q, q_out=qr)
                N.attention_pages(pages, b, qr, out, frame_tokens=frame, window=window)
            N.gate_norm(x, out @ w[1], x_out, h_out, pre=pre, post=post, mod=mod)
        return run, x_out, h_out
    grid = lambda p: torch.stack([p // frame, p % frame // gw, p % frame % gw], 1).int()
    at = [torch.arange(t, device="cuda") for t in total]
    prompt = torch.cat([x[:f * frame] for x, f in zip(xs, frames)])
    run, px, ph = step(prompt, [f * frame for f in frames], torch.cat([grid(a[:f * frame]) for a, f in zip(at, frames)]), True)
    run()
    last = torch.cat([x[-frame:] for x in xs])
    run2, fx, fh = step(last, [frame, frame], None, False)
    kv_len += frame
    run2()                                                             # (first calls outside the capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run2()
    fx.zero_(), fh.zero_()
    graph.replay()
    parts = mods.split(width, 1)
    p0 = f0 = 0
    for s, (x, f) in enumerate(zip(xs, frames)):
        row = [m.expand(x.shape[0], -1) for m in parts]
        want_x, want_h = _block64(x, w, row, "rms", rope, grid(at[s]), [(0, x.shape[0])], heads, share, dh, frame, window)
        n = f * frame
        for got, want in ((px[p0:p0 + n], want_x[:n]), (fx[f0:f0 + frame], want_x[n:]), (ph[p0:p0 + n], want_h[:n]), (fh[f0:f0 + frame], want_h[n:])):
            # bf16 roundings on the way, relative to their tensors: h, q, k and v before and after the rotation, P, out, the projection, h: about
            # ten of at most 2^-8 each
            assert ((got.double() - want).norm() / want.norm()) < 10 * 2.0 ** -8
        p0, f0 = p0 + n, f0 + frame


def test_calls_on_other_streams_overlap():
    """No working memory: calls on two streams at once and on a stream that is not torch's current one give what they give alone."""
    torch, N = _mods()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    n = 1500
    q, k, v = (torch.randn(n, 4, 64, device="cuda").bfloat16() for _ in range(3))
    b = N.Batch(n, row_start=_int([0, 700, n]), max_rows=800)
    alone = torch.zeros(n, 256, device="cuda", dtype=torch.bfloat16)
    N.attention_packed(b, q, k, v, alone)
    outs = [torch.zeros_like(alone) for _ in range(8)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        N.attention_packed(b, q, k, v, o, stream=(s1, s2)[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, alone) for o in outs)


def test_captured_calls_follow_lengths_and_tables():
    """A captured call reads lengths, row starts and tables when it runs."""
    torch, N = _mods()
    pages = N.Pages(*(torch.randn(30, 2, 32, 64, device="cuda").bfloat16() for _ in range(2)))
    kv, start, table = _int([500, 300]), _int([0, 90, 100]), torch.randperm(30, device="cuda")[:30].view(2, 15).int()
    q = torch.randn(200, 4, 64, device="cuda").bfloat16()
    out = torch.zeros(200, 256, device="cuda", dtype=torch.bfloat16)
    b = N.Batch(200, kv, table=table, row_start=start, max_rows=150)
    run = lambda: N.attention_pages(pages, b, q, out)
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rows, lens in (([90, 10], [500, 300]), ([1, 150], [480, 200]), ([0, 0], [5, 5]), ([150, 50], [150, 480])):
        kv.copy_(_int(lens)), start.copy_(_int([0, rows[0], sum(rows)])), table.copy_(table.flip(0).clone())
        out.fill_(7.0)
        run()
        direct = out.clone()
        out.fill_(7.0)
        graph.replay()
        assert torch.equal(out, direct) and (out[sum(rows):] == 7).all()


def test_what_the_device_says_is_clamped():
    """Row starts and lengths with nonsense in them: nothing is written outside the row buffers' live part, a good sequence is right."""
    torch, N = _mods()
    q, k, v = (torch.randn(64, 2, 64, device="cuda").bfloat16() for _ in range(3))
    for rows in (4, 64):
        good, out = (torch.full((64, 128), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        N.attention_packed(N.Batch(64, row_start=_int([0, rows]), max_rows=rows), q, k, v, good)
        N.attention_packed(N.Batch(64, row_start=_int([-5, rows, 1 << 30, -1, -(1 << 31)]), max_rows=rows), q, k, v, out)
        assert torch.equal(out[:rows], good[:rows])
    pages = N.Pages(*(torch.randn(8, 2, 16, 64, device="cuda").bfloat16() for _ in range(2)))
    out = torch.zeros(64, 128, device="cuda", dtype=torch.bfloat16)
    for big in (4, 64):
        b = N.Batch(64, _int([-7, (1 << 31) - 1, 100]), _int([[0, 1 << 30], [-1, 99], [1, 2]]), row_start=_int([0, 5, 9, 64]), max_rows=big)
        N.attention_pages(pages, b, q, out)
    torch.cuda.synchronize()
