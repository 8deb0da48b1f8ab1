"""What the calls around a block's projections refuse.  No GPU: every check comes before the first CUDA call, and the pointers
are never followed."""
import ctypes as C
import os
import re

import pytest

from paper_2506_01380_b200 import inputs as I
from paper_2506_01380_b200 import nfd as N
from tests.test_paged_refusals import A, ALIGN, BADCFG, BATCHES, NULLPTR, PAGED, PAGES, RANGE, _batch, _pages, _ref, _rope


def pages(p=_pages(dtype=1), batch=_batch(), heads=4, q=A, qs=256, frame=12, window=2, out=A):
    return N.load().nfd_attention_pages(_ref(p), _ref(batch), heads, q, qs, frame, window, out, None)


def packed(batch=_batch(kv_len=None, table=None, table_len=0), dtype=1, heads=4, kv_heads=2, dh=64, q=A, qs=256, k=A, ks=128, v=A, vs=128,
           frame=12, window=2, out=A):
    return N.load().nfd_attention_packed(_ref(batch), dtype, heads, kv_heads, dh, q, qs, k, ks, v, vs, frame, window, out, None)


def rotate(rope=_rope(), flags=0, dtype=1, dh=64, n=8, pos=A, h=2, x=A, xs=128, xo=A, xos=128, h2=1, y=A, ys=64, yo=A, yos=64):
    return N.load().nfd_rotate(_ref(rope), flags, dtype, dh, n, pos, h, x, xs, xo, xos, h2, y, ys, yo, yos, None)


def _norm(**kw):
    d = dict(kind=0, dtype=0, eps=1e-6, weight=A, bias=A)
    d.update(kw)
    return N.NfdNorm(*[d[n] for n, _ in N.NfdNorm._fields_])


def _mod(**kw):
    d = dict(gate=A, scale=A, shift=A, stride=128, index=A, n_mods=3, rows_per_mod=0, dtype=0)
    d.update(kw)
    return N.NfdModulation(*[d[n] for n, _ in N.NfdModulation._fields_])


def norm(n=4, width=128, xt=0, x=A, xs=128, dtype=1, y=A, ys=128, xo=A, xos=128, h=A, hs=128, post=_norm(), pre=_norm(), mod=_mod(), res=1.0):
    return N.load().nfd_gate_norm(n, width, xt, x, xs, dtype, y, ys, xo, xos, h, hs, _ref(post), _ref(pre), _ref(mod), res, None)


def test_pages_refuses():
    for code, b in PAGED:
        assert pages(batch=b) == code, code
    for code, p in PAGES:
        assert pages(p=p) == code, code
    assert pages(p=_pages()) == BADCFG                                 # 4-bit pages have a call of their own
    for code, kw in [(NULLPTR, dict(q=None)), (NULLPTR, dict(out=None)), (ALIGN, dict(q=A + 2)), (ALIGN, dict(out=A + 8)),
                     (ALIGN, dict(qs=260)), (RANGE, dict(qs=128)), (RANGE, dict(heads=3)), (RANGE, dict(heads=0)),
                     (RANGE, dict(heads=2048)), (RANGE, dict(frame=0)), (RANGE, dict(frame=(1 << 20) + 1)), (RANGE, dict(window=-1)),
                     (RANGE, dict(batch=_batch(n_rows=1 << 30, max_rows=1 << 30)))]:
        assert pages(**kw) == code, (code, kw)


def test_packed_refuses():
    for code, b in BATCHES:
        if b is None or b.kv_len in (A, None):                         # (lengths and tables are not looked at)
            assert packed(batch=b) == code, code
    for code, kw in [(NULLPTR, dict(q=None)), (NULLPTR, dict(k=None)), (NULLPTR, dict(v=None)), (NULLPTR, dict(out=None)),
                     (ALIGN, dict(q=A + 2)), (ALIGN, dict(k=A + 8)), (ALIGN, dict(v=A + 4)), (ALIGN, dict(out=A + 8)),
                     (ALIGN, dict(qs=260)), (ALIGN, dict(ks=132)), (RANGE, dict(qs=128)), (RANGE, dict(ks=64)), (RANGE, dict(vs=-128)),
                     (RANGE, dict(heads=3)), (RANGE, dict(kv_heads=0)), (RANGE, dict(heads=0)), (RANGE, dict(heads=2048)),
                     (BADCFG, dict(dtype=2)), (BADCFG, dict(dh=96)), (BADCFG, dict(dh=0)), (RANGE, dict(frame=0)), (RANGE, dict(window=-1)),
                     (RANGE, dict(batch=_batch(n_rows=1 << 30, max_rows=1 << 30)))]:
        assert packed(**kw) == code, (code, kw)


def test_rotate_refuses():
    for code, kw in [(NULLPTR, dict(rope=None)), (BADCFG, dict(flags=4)), (BADCFG, dict(dtype=2)), (BADCFG, dict(dh=72)), (BADCFG, dict(dh=272)),
                     (BADCFG, dict(dh=0)), (BADCFG, dict(rope=_rope(rope_t=18))), (BADCFG, dict(rope=_rope(rope_t=15, rope_h=25))),
                     (BADCFG, dict(rope=_rope(rope_t=-2, rope_h=42))), (BADCFG, dict(rope=_rope(theta=0.0))),
                     (BADCFG, dict(rope=_rope(theta=float("nan")))), (RANGE, dict(n=-1)), (RANGE, dict(n=(1 << 30) + 1)),
                     (RANGE, dict(h=-1)), (RANGE, dict(h2=1025)), (ALIGN, dict(pos=A + 2)), (NULLPTR, dict(pos=None)),
                     (NULLPTR, dict(x=None)), (NULLPTR, dict(xo=None)), (NULLPTR, dict(y=None)), (ALIGN, dict(x=A + 8)), (ALIGN, dict(yo=A + 2)),
                     (ALIGN, dict(xs=129)), (RANGE, dict(xs=64)), (RANGE, dict(yos=32)), (BADCFG, dict(xs=256)), (BADCFG, dict(yos=128))]:
        assert rotate(**kw) == code, (code, kw)


def test_gate_norm_refuses():
    for code, kw in [(BADCFG, dict(xt=2)), (BADCFG, dict(dtype=2)), (RANGE, dict(n=-1)), (RANGE, dict(width=0)), (RANGE, dict(width=124)),
                     (RANGE, dict(width=16392)), (NULLPTR, dict(x=None)), (NULLPTR, dict(xo=None)), (NULLPTR, dict(pre=None)),
                     (ALIGN, dict(x=A + 8)), (ALIGN, dict(y=A + 2)), (ALIGN, dict(xo=A + 8)), (ALIGN, dict(h=A + 8)), (ALIGN, dict(xs=129)),
                     (RANGE, dict(xs=120)), (RANGE, dict(ys=64)), (RANGE, dict(hs=-128)), (BADCFG, dict(xos=256)), (BADCFG, dict(hs=256)),
                     (BADCFG, dict(pre=_norm(kind=2))), (BADCFG, dict(post=_norm(dtype=2))), (BADCFG, dict(post=_norm(eps=-1.0))),
                     (BADCFG, dict(pre=_norm(eps=float("nan")))), (ALIGN, dict(pre=_norm(weight=A + 4))), (ALIGN, dict(post=_norm(bias=A + 8))),
                     (BADCFG, dict(mod=_mod(dtype=2))), (RANGE, dict(mod=_mod(n_mods=0))), (RANGE, dict(mod=_mod(index=None))),
                     (RANGE, dict(mod=_mod(stride=64))), (ALIGN, dict(mod=_mod(stride=130))), (ALIGN, dict(mod=_mod(gate=A + 8))),
                     (ALIGN, dict(mod=_mod(index=A + 2)))]:
        assert norm(**kw) == code, (code, kw)


def test_calls_without_rows_do_nothing_and_need_no_buffers():
    """(Without a GPU a launch would fail.)"""
    none = _batch(n_rows=0, max_rows=0)
    assert pages(batch=none, q=None, out=None) == 0
    assert packed(batch=none, q=None, k=None, v=None, out=None) == 0
    assert rotate(n=0, pos=None, x=None, xo=None, y=None, yo=None) == 0 and rotate(h=0, h2=0, pos=None) == 0
    assert norm(n=0, x=None, y=None, xo=None, h=None) == 0 and norm(y=None, h=None) == 0
    assert pages(batch=none, q=A + 2) == ALIGN and packed(batch=none, ks=100) == ALIGN


@pytest.mark.parametrize("name,struct", [("nfd_norm", N.NfdNorm), ("nfd_modulation", N.NfdModulation)])
def test_structs_match_header(name, struct):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "nfd.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.findall(r"typedef struct \{([^{}]*)\} %s;" % name, text)[0]
    got = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        kind = C.c_void_p if "*" in decl else {"int": C.c_int, "float": C.c_float, "long long": C.c_longlong}[
            re.match(r"(long long|int|float)", re.sub(r"^const ", "", decl)).group(1)]
        got += [(n.strip(), kind) for n in re.sub(r"^(const |unsigned |long long |int |float |char |void )+", "", decl)
                .replace("*", "").split(",")]
    assert got == list(struct._fields_), name
    for const in ("NORM_LAYER", "NORM_RMS", "ROTATE_HALVES", "ROTATE_BACK"):
        assert int(re.search(r"#define NFD_%s (\d+)" % const, text).group(1)) == getattr(I, const)
