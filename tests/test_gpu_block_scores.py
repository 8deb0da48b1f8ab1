"""Scores far apart in the attention to pages and packed prompts, of many rows to bf16 keys above all, against the 64-bit oracle: one key far above or below the others, at each place of the
sixteen columns that are taken at a time; a key that is not a number.

Bounds: as in test_gpu_block.py, with 1.2e-4 more of a probability for those exponentials that are polynomials (1.0e-4, and 1.6e-5 of their arguments).
"""
import numpy as np
import pytest

from oracle import block_oracle as O
from test_gpu_block import EVER, HALF, _batch, _int, _mods, _randn, _smax

pytestmark = pytest.mark.gpu

PLACES = 16                                                # a head of keys each
ABOVE = [60, 120, 130, 150, 170, 185, 250, 330, 390]       # a sequence each, the score, of which probabilities are the exponential
CALLS = [("boxes", 1, 3), ("odd pages", 4, 2), ("boxes", 1, 150), ("boxes", 1, 400), ("boxes", 4, 40), ("odd pages", 1, 150), ("odd pages", 4, 110), ("packed", 1, 0), ("packed", 2, 0)]
POLY = 1.2e-4


def _close(got, want, mag, smax, n, dh, half=HALF):
    torch, _ = _mods()
    e = (dh + 4) * 2.0 ** -23 * smax + 2.0 ** -21 + (POLY if half else 0.0)
    bound = (2 * e + n * 2.0 ** -23 + 1.01 * half) * mag + (1.01 * half if half else 2.0 ** -23) * want.abs() + 1e-30
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan)
    assert ((got.double() - want).abs() <= bound)[~nan].all(), torch.where(nan, 0.0, (got.double() - want).abs() - bound).max().item()


def _check(kind, dh, share, rows, length, poke, n_seqs, window=EVER, seed=0, dtype="bfloat16"):
    """n_seqs sequences of `length` tokens, PLACES heads of keys; the rows are the last `rows` of them (packed: all).  poke(q, k, v) has q [seqs, rows, heads of
    keys, share, dh] and k, v [seqs, length, heads of keys, dh] with ordinary numbers in them."""
    torch, N = _mods()
    dt = getattr(torch, dtype)
    g = torch.Generator("cuda").manual_seed(seed)
    rows = length if kind == "packed" else rows
    q = _randn(g, n_seqs, rows, PLACES, share, dh, dtype=torch.float32) * 0.3
    k = _randn(g, n_seqs, length, PLACES, dh, dtype=torch.float32) * 0.3
    v = _randn(g, n_seqs, length, PLACES, dh, dtype=torch.float32)
    poke(q, k, v)
    q, k, v = q.flatten(2, 3).to(dt), k.to(dt), v.to(dt)
    out = torch.full((n_seqs * rows, PLACES * share * dh), 7.0, device="cuda", dtype=dt)
    if kind == "packed":
        b, _, _ = _batch([rows] * n_seqs)
        N.attention_packed(b, q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), out, window=window)
    else:
        page = 64 if kind == "boxes" else 50
        per = -(-length // page)
        table = torch.randperm(n_seqs * per, generator=g, device="cuda").view(n_seqs, per)
        pages = []
        for t in (k, v):
            t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, per * page - length)).unflatten(1, (per, page)).transpose(2, 3)
            p = torch.empty(n_seqs * per, PLACES, page, dh, device="cuda", dtype=dt)
            p[table.flatten()] = t.flatten(0, 1)
            pages.append(p)
        b, _, _ = _batch([rows] * n_seqs, [length] * n_seqs, table.int())
        N.attention_pages(N.Pages(*pages), b, q.flatten(0, 1), out, window=window)
    got = out.view(n_seqs, rows, PLACES * share, dh)
    seen = O.seen_tokens(rows, length, 1, window)
    for s in range(n_seqs):
        want, mag = O.attend(q[s], k[s], v[s], seen)
        _close(got[s], want, mag, _smax(q[s], k[s]), length, dh, HALF if dtype == "bfloat16" else 0.0)


def _lone(above):
    """Key 288 + place (in the middle of the blocks; their columns are tokens modulo 16) `above` over the others, with a value of its own."""
    def poke(q, k, v):
        dh = q.shape[-1]
        q[..., 0], k[..., 0] = 16.0, 0.0
        for s, a in enumerate(above):
            for place in range(PLACES):
                k[s, 288 + place, place, 0] = a * dh ** 0.5 / 16
        v[:, 288:304] = 5.0
    return poke


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("kind,share,rows", CALLS)
def test_one_key_far_above_the_others(kind, dh, share, rows):
    """A call of all of them, and (keys split over clusters) of one sequence at a time."""
    _check(kind, dh, share, rows, 800, _lone(ABOVE), len(ABOVE))
    _check(kind, dh, share, rows, 800, _lone(ABOVE), len(ABOVE), dtype="float32")
    for a in ABOVE if share == 1 else ABOVE[3:4]:
        _check(kind, dh, share, rows, 1500, _lone([a]), 1)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("kind,share,rows", CALLS)
def test_a_first_key_far_above_the_others(kind, dh, share, rows):
    """What a first token that takes most of the weight leaves the rest: 200 and 60 above, and 45, where theirs is still in the sums; beside the largest values there are, which
    must not show where their probability is nothing."""
    above = [200.0, 60.0, 45.0]

    def poke(q, k, v):
        q[..., 0], k[..., 0] = 16.0, 0.0
        for s, a in enumerate(above):
            k[s, 0, :, 0] = a * dh ** 0.5 / 16
        v[0, 290:420:3] = 3e38
        v[0, 291:420:3] = -3e38
    _check(kind, dh, share, rows, 800, poke, len(above))


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("kind,share,rows", CALLS)
def test_scores_spread_over_a_hundred(kind, dh, share, rows):
    def poke(q, k, v):
        q *= 10
        k *= 10
    _check(kind, dh, share, rows, 800, poke, 3)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("kind,share,rows", CALLS)
def test_a_seen_key_that_is_not_a_number(kind, dh, share, rows):
    """In one place of sixteen for each head, in a block that all rows of a tile see and in one that some do: the rows that see it are NaN, and no others."""
    def poke(q, k, v):
        for place in range(PLACES):
            k[0, 288 + place, place, 3] = float("nan")
            k[1, 740 + place, place, 3] = float("nan")
    for dtype in ("bfloat16", "float32"):
        _check(kind, dh, share, rows, 800, poke, 3, dtype=dtype)
        _check(kind, dh, share, rows, 800, poke, 3, window=400, dtype=dtype)


@pytest.mark.parametrize("dh,part,page,pages,rows", [(128, 64, 64, 4, 40), (64, 96, 32, 12, 80), (32, 96, 32, 12, 80)])
@pytest.mark.parametrize("share", [1, 4])
def test_sums_that_have_grown_in_every_part_stay_finite(dh, part, page, pages, rows, share):
    """What a sum may grow by before its reference follows, in each part of a row's keys, which a ring of pages has begin inside one: keys of a power of two of
    parts, in one part more.  The values are as large as they go, and so is their mean."""
    torch, N = _mods()
    held, shift = page * pages, 8
    length = held + shift
    growth = torch.zeros(length, dtype=torch.float64)
    for a in range(0, length, part):
        growth[a + 16:a + part] = 50 - np.log2(part - 16) - 0.02       # (the first sixteen are the reference where it is the row's first part)
    growth[held:] = 50 - np.log2(shift) - 0.02
    c = np.log2(np.e) / np.sqrt(dh)
    score = growth / c                                                 # as 2 k0 + k1 / 16, of bf16 numbers
    k0 = (score / 2).floor()
    kk = torch.zeros(length, 1, dh, dtype=torch.float64)
    kk[:, 0, 0], kk[:, 0, 1] = k0.bfloat16().double(), ((score - 2 * k0.bfloat16().double()) * 16).bfloat16().double()
    big = torch.finfo(torch.bfloat16).max * 0.99
    kk, vv = kk.bfloat16().cuda(), torch.full((length, 1, dh), big, device="cuda").bfloat16()
    k, v = (torch.zeros(pages, 1, page, dh, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    t = np.arange(length)[shift:]
    k[t // page % pages, :, t % page], v[t // page % pages, :, t % page] = kk[shift:], vv[shift:]
    q = torch.zeros(rows, share, dh, device="cuda", dtype=torch.bfloat16)
    q[..., 0], q[..., 1] = 2.0, 1 / 16
    out = torch.zeros(rows, share * dh, device="cuda", dtype=torch.bfloat16)
    b, _, _ = _batch([rows], [length], _int(np.arange(pages)[None]))
    N.attention_pages(N.Pages(k, v), b, q, out)
    got = out.view(rows, share, dh)
    want, mag = O.attend(q, kk[shift:], vv[shift:], O.seen_tokens(rows, length, 1, EVER)[:, shift:])
    s = 2.0 ** -100
    assert torch.isfinite(got).all()
    _close(got.double() * s, want * s, mag * s, _smax(q, kk), length, dh)


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("kind,share,rows", CALLS)
def test_scores_that_are_not_finite(kind, dh, share, rows):
    """A score of -inf is a probability of 0, one of inf none at all: the rows that see it are NaN; a query that is not a number is its own row's affair."""
    def poke(q, k, v):
        q[..., 3] = q[..., 3].abs() + 0.1
        for place in range(PLACES):
            k[0, 288 + place, place, 3] = float("-inf")
            k[1, 288 + place, place, 3] = float("inf")
        q[2, q.shape[1] // 2, 5, 0, 7] = float("nan")
    for dtype in ("bfloat16", "float32"):
        _check(kind, dh, share, rows, 800, poke, 3, dtype=dtype)
