"""The calls on the caller's own memory at the ends of their numbers' ranges.  Bounds as in test_gpu_paged.py."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import paged_oracle as P
from test_gpu_paged import HALF, _largest_score, _mods, _np, _rounded, _within

pytestmark = pytest.mark.gpu


def _states_case(tdt, seqs, rows, keys, dh, power, scores, seed):
    """States whose values have a size of 2^power, and queries whose scores are a function of the key's number (in nats): everything 64 bits
    needs to judge the call, and its result."""
    torch, N = _mods()
    rng = np.random.default_rng(seed)
    k = rng.standard_normal((seqs, keys, 1, dh)).astype(np.float32)
    q = np.zeros((seqs * rows, 1, dh), np.float32)
    q[..., 0], q[..., 1] = np.sqrt(dh), 1.0                            # (and a little of another channel)
    k[..., 0] = scores[None, :, None]
    v = rng.uniform(-1.9, 1.9, k.shape)
    k, q = _rounded(k, tdt), _rounded(q, tdt)
    v = (_rounded(v.astype(np.float32), tdt).double() * 2.0 ** power).to(tdt)
    assert torch.isfinite(v).all()
    b = N.Batch(seqs * rows, n_seqs=seqs)
    out = torch.full((seqs * rows, dh), 7.0, device="cuda", dtype=tdt)
    N.cross_attention(N.States(k.cuda(), v.cuda()), b, q.cuda(), out)
    batch = dict(rows=[rows] * seqs, lens=[keys] * seqs)
    want, mag = P.cross_attention(_np(q), batch, _np(k), _np(v).astype(np.float64), None, 1)
    return out, want, mag, _largest_score(_np(q), _np(k))


RISES = {"equal": lambda n: np.zeros(n, np.float32),
         "rising by 41": lambda n: np.where(np.arange(n) < 16, 0, 41 * np.arange(n) / n).astype(np.float32),
         "late": lambda n: np.where(np.arange(n) < n - 3, 0, 30).astype(np.float32)}


@pytest.mark.parametrize("power", [100, 127, -90])
@pytest.mark.parametrize("scores", list(RISES))
@pytest.mark.parametrize("seqs,rows", [(1, 1), (3, 24), (1, 140), (150, 300)])
@pytest.mark.parametrize("tdt,dh", [("bfloat16", 64), ("bfloat16", 128), ("float32", 64)])
def test_cross_large_and_small_values(tdt, dh, seqs, rows, scores, power):
    """Results are means of the values: finite where these are, however the scores rise, for every number of rows."""
    torch, _ = _mods()
    if seqs > 100 and tdt == "float32":
        seqs = 5                                                       # (many sequences are for the layouts of the bf16 kernel)
    keys = 700
    out, want, mag, smax = _states_case(getattr(torch, tdt), seqs, rows, keys, dh, power, RISES[scores](keys), rows)
    s = 2.0 ** -power
    _within(_np(out).astype(np.float64).reshape(want.shape) * s, want * s, mag * s, smax, keys, HALF if tdt == "bfloat16" else 0.0)


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [0, 90, 699])
@pytest.mark.parametrize("seqs,rows", [(1, 1), (3, 24), (1, 140), (1, 336), (150, 300)])
@pytest.mark.parametrize("tdt,dh", [("bfloat16", 64), ("bfloat16", 128), ("float32", 64)])
def test_cross_values_that_are_not_finite(tdt, dh, seqs, rows, at, what):
    """A value that is not finite makes its column of the rows that see it not finite, however small the probability: here the scores of
    later keys are 120 nats above those of earlier ones.  Other columns hold."""
    torch, N = _mods()
    dt = getattr(torch, tdt)
    keys, g = 700, torch.Generator("cuda").manual_seed(rows)
    k, v = (torch.randn(seqs, keys, 1, dh, device="cuda", generator=g).to(dt) for _ in range(2))
    k[..., 0] = torch.where(torch.arange(keys, device="cuda") < 100, 0.0, 120.0)[None, :, None].to(dt)
    q = torch.zeros(seqs * rows, 1, dh, device="cuda", dtype=dt)
    q[..., 0], q[..., 1] = dh ** 0.5, 1.0
    b = N.Batch(seqs * rows, n_seqs=seqs)
    run = lambda vv: N.cross_attention(N.States(k, vv), b, q, torch.full((seqs * rows, dh), 7.0, device="cuda", dtype=dt))
    good, bad = run(v), v.clone()
    bad[:, at, 0, 5] = what
    got = run(bad)
    assert not got[:, 5].isfinite().any()
    rest = torch.arange(dh, device="cuda") != 5
    assert good.isfinite().all() and torch.equal(got[:, rest], good[:, rest])


# ---------------------------------------------------------------------------------------------------------------
# 4-bit numbers
# ---------------------------------------------------------------------------------------------------------------
def _step(lo, hi):
    """The smallest number of 4 significant bits, at least 2^-100, with 15 of it at least hi - lo, in fractions."""
    r, e = Fraction(float(hi)) - Fraction(float(lo)), -100
    while Fraction(2) ** e * 15 * 15 / 8 < r:
        e += 1
    return next(float(Fraction(2) ** e * m / 8) for m in range(8, 16) if Fraction(2) ** e * m / 8 * 15 >= r)


@pytest.mark.parametrize("hi,lo", [(15.0, -1e-8), (15.0, -1e-30), (1e-9, -15.0), (15.0, 0.0), (30.0 - 2.0 ** -19, -2.0 ** -19), (7.5, -7.5 - 2.0 ** -21),
                                   (16.875 * 2.0 ** 40, -1.0)])
def test_append_steps_by_the_definition(hi, lo):
    """Ranges that lie next to 15 steps: what fp32 rounds away of hi - lo decides."""
    torch, N = _mods()
    x = torch.zeros(1, 1, 64)
    x[0, 0, 3], x[0, 0, 9], x[0, 0, 32:] = hi, lo, torch.linspace(-1, 1, 32)
    hi, lo = float(x[0, 0, 3]), float(x[0, 0, 9])
    pages = N.Pages.empty("kv4", 1, 1, 1, 64)
    b = N.Batch(1, torch.ones(1, device="cuda", dtype=torch.int32), torch.zeros(1, 1, device="cuda", dtype=torch.int32))
    N.kv_append(pages, b, x.cuda(), x.cuda())
    step = _step(lo, hi)
    for words in (pages.k_scale, pages.v_scale):
        w = int(words[0, 0, 0, 0]) & 0xFFFF
        got = float(np.uint32((w & 0xFFF0) << 16).view(np.float32))
        assert got == step and w & 15 == round(Fraction(-lo) / Fraction(step))


@pytest.mark.parametrize("rows", [1, 150])
@pytest.mark.parametrize("power", [-100, -99, -98, -97, -94])
def test_kv4_smallest_steps(rows, power):
    """Steps from 2^-98 on are taken as they are; a value of a smaller one to within 2^-101 (half of it by the zero, half by the number)."""
    torch, N = _mods()
    rng = np.random.default_rng(12)
    t = lambda a: torch.as_tensor(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()
    x = rng.standard_normal((4, 1, 64, 64)).astype(np.float32)
    (kb, kw), (vb, vw) = P.kv4_bytes(*P.kv4_quantise(x)), P.kv4_bytes(*P.kv4_quantise(x[::-1].copy()))
    vw = ((vw & 0x7F) | ((127 + power) << 7)).astype(np.uint16)        # (steps of 4 bits, as they come)
    b = N.Batch(rows, torch.tensor([256], device="cuda", dtype=torch.int32), torch.arange(4, device="cuda", dtype=torch.int32)[None])
    q = _np(_rounded(rng.standard_normal((rows, 1, 64)).astype(np.float32), torch.bfloat16))
    out = torch.zeros(rows, 64, device="cuda", dtype=torch.bfloat16)
    N.attention_kv4(N.Pages(t(kb), t(vb), t(kw), t(vw)), b, torch.as_tensor(q).cuda().bfloat16(), out)
    want, mag = P.attention_kv4(q, dict(rows=[rows], lens=[256]), np.arange(4)[None], (kb, kw, vb, vw), 1, 1 << 30, 1)
    off = np.abs(_np(out).astype(np.float64).reshape(rows, 1, 64) - want)
    # (2^-109: 256 sums of numbers scaled by 2^-32 that may be below fp32's normal ones, to 2^-149 each)
    bound = (2.0 ** -101 if power < -98 else 0) + 2.0 ** -109 + 1.02 * HALF * (mag + np.abs(want))
    assert (off <= bound).all(), float((off / bound).max())
