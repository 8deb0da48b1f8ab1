"""What the calls on the caller's own memory refuse, and the oracle's 4-bit numbers.  No GPU: every check comes before the
first CUDA call, and the pointers are never followed."""
import ctypes as C

import numpy as np
import pytest

from oracle import paged_oracle as P
from paper_2506_01380_b200 import inputs as I
from paper_2506_01380_b200 import nfd as N

A = 0x10000          # an aligned address that nothing reads
BADCFG, NULLPTR, ALIGN, RANGE = -1, -2, -3, -4


def _batch(**kw):
    d = dict(row_start=A, kv_len=A, table=A, n_seqs=2, n_rows=8, max_rows=4, table_len=3)
    d.update(kw)
    return N.NfdBatch(*[d[n] for n, _ in N.NfdBatch._fields_])


def _pages(**kw):
    d = dict(k=A, v=A, k_scale=A, v_scale=A, dtype=I.DTYPE_KV4, n_pages=4, n_heads=2, page_tokens=16, head_dim=64)
    d.update(kw)
    return N.NfdPages(*[d[n] for n, _ in N.NfdPages._fields_])


def _rope(**kw):
    d = dict(rope_t=16, rope_h=24, rope_w=24, theta=1e4, frame_tokens=12, grid_w=4)
    d.update(kw)
    return N.NfdRope(*[d[n] for n, _ in N.NfdRope._fields_])


def _states(**kw):
    d = dict(k=A, v=A, mask=None, seq_stride=1024, key_stride=128, head_stride=64, dtype=I.DTYPE_BF16, n_keys=8, n_heads=2,
             head_dim=64)
    d.update(kw)
    return N.NfdStates(*[d[n] for n, _ in N.NfdStates._fields_])


def _ref(c):
    return C.byref(c) if c is not None else None


def append(pages=_pages(), batch=_batch(), rope=_rope(), dtype=1, k=A, ks=128, v=A, vs=128, hq=4, q=A, qs=256, q_out=A):
    return N.load().nfd_kv_append(_ref(pages), _ref(batch), _ref(rope), dtype, k, ks, v, vs, hq, q, qs, q_out, None)


def read(pages=_pages(), batch=_batch(), dtype=1, k=A, v=A):
    return N.load().nfd_pages_read(_ref(pages), _ref(batch), dtype, k, v, None)


def kv4(pages=_pages(), batch=_batch(), heads=4, q=A, qs=256, frame=12, window=2, out=A):
    return N.load().nfd_attention_kv4(_ref(pages), _ref(batch), heads, q, qs, frame, window, out, None)


def cross(states=_states(), batch=_batch(), heads=4, q=A, qs=256, out=A):
    return N.load().nfd_cross_attention(_ref(states), _ref(batch), heads, q, qs, out, None)


BATCHES = [(NULLPTR, None), (RANGE, _batch(n_seqs=0)), (RANGE, _batch(n_seqs=65536)), (RANGE, _batch(n_rows=-1)),
           (RANGE, _batch(max_rows=9)), (RANGE, _batch(max_rows=-1)), (RANGE, _batch(row_start=None, max_rows=3)),
           (ALIGN, _batch(row_start=A + 2)), (ALIGN, _batch(kv_len=A + 1))]
PAGED = BATCHES + [(NULLPTR, _batch(kv_len=None)), (NULLPTR, _batch(table=None)), (RANGE, _batch(table_len=0)),
                   (ALIGN, _batch(table=A + 2))]
PAGES = [(NULLPTR, None), (NULLPTR, _pages(k=None)), (NULLPTR, _pages(v=None)), (NULLPTR, _pages(k_scale=None)),
         (NULLPTR, _pages(v_scale=None)), (BADCFG, _pages(dtype=3)), (BADCFG, _pages(dtype=-1)), (BADCFG, _pages(head_dim=48)),
         (ALIGN, _pages(k=A + 8)), (ALIGN, _pages(v_scale=A + 2)), (RANGE, _pages(n_pages=0)), (RANGE, _pages(n_heads=0)),
         (RANGE, _pages(n_heads=1025)), (RANGE, _pages(page_tokens=0)), (RANGE, _pages(page_tokens=(1 << 20) + 1))]


@pytest.mark.parametrize("call", [append, read, kv4])
def test_paged_calls_refuse_bad_caches_and_batches(call):
    for code, b in PAGED:
        assert call(batch=b) == code, (code, [(n, getattr(b, n)) for n, _ in N.NfdBatch._fields_] if b else None)
    for code, p in PAGES:
        assert call(pages=p) == code, (code, [(n, getattr(p, n)) for n, _ in N.NfdPages._fields_] if p else None)


def test_append_refuses():
    for code, kw in [(NULLPTR, dict(k=None)), (NULLPTR, dict(v=None)), (NULLPTR, dict(q=None)), (NULLPTR, dict(q_out=None)),
                     (ALIGN, dict(k=A + 8)), (ALIGN, dict(q_out=A + 4)), (ALIGN, dict(ks=129)), (ALIGN, dict(qs=257)),
                     (RANGE, dict(ks=64)), (RANGE, dict(vs=-128)), (RANGE, dict(hq=-1)), (RANGE, dict(hq=1025)),
                     (BADCFG, dict(dtype=2)), (BADCFG, dict(pages=_pages(dtype=0))), (BADCFG, dict(pages=_pages(dtype=1), dtype=0)),
                     (BADCFG, dict(rope=_rope(rope_t=18))), (BADCFG, dict(rope=_rope(rope_t=15, rope_h=25))),
                     (BADCFG, dict(rope=_rope(rope_t=-2, rope_h=42))), (BADCFG, dict(rope=_rope(theta=0.0))),
                     (BADCFG, dict(rope=_rope(theta=float("inf")))), (BADCFG, dict(rope=_rope(theta=float("nan")))),
                     (BADCFG, dict(rope=_rope(frame_tokens=0))), (BADCFG, dict(rope=_rope(grid_w=5)))]:
        assert append(**kw) == code, (code, kw)


def test_read_refuses():
    for code, kw in [(BADCFG, dict(dtype=2)), (BADCFG, dict(pages=_pages(dtype=0))), (ALIGN, dict(k=A + 8)), (ALIGN, dict(v=A + 8))]:
        assert read(**kw) == code, (code, kw)


def test_kv4_attention_refuses():
    for code, kw in [(NULLPTR, dict(q=None)), (NULLPTR, dict(out=None)), (ALIGN, dict(q=A + 2)), (ALIGN, dict(out=A + 8)),
                     (ALIGN, dict(qs=260)), (RANGE, dict(qs=128)), (RANGE, dict(heads=3)), (RANGE, dict(heads=0)),
                     (RANGE, dict(heads=2048)), (RANGE, dict(frame=0)), (RANGE, dict(frame=(1 << 20) + 1)), (RANGE, dict(window=-1)),
                     (BADCFG, dict(pages=_pages(dtype=1))),
                     (RANGE, dict(batch=_batch(n_rows=1 << 21, max_rows=1 << 20))),
                     (RANGE, dict(batch=_batch(n_rows=1 << 30, max_rows=1 << 30)))]:
        assert kv4(**kw) == code, (code, kw)


def test_cross_attention_refuses():
    for code, b in BATCHES:
        assert cross(batch=b) == code
    for code, kw in [(NULLPTR, dict(states=None)), (NULLPTR, dict(states=_states(k=None))), (NULLPTR, dict(states=_states(v=None))),
                     (BADCFG, dict(states=_states(dtype=2))), (BADCFG, dict(states=_states(head_dim=96))),
                     (RANGE, dict(states=_states(n_keys=-1))), (RANGE, dict(states=_states(n_heads=0))),
                     (RANGE, dict(states=_states(key_stride=-128))), (ALIGN, dict(states=_states(key_stride=132))),
                     (ALIGN, dict(states=_states(seq_stride=1020))), (ALIGN, dict(states=_states(k=A + 8))),
                     (NULLPTR, dict(q=None)), (NULLPTR, dict(out=None)), (ALIGN, dict(q=A + 2)), (RANGE, dict(qs=128)),
                     (RANGE, dict(heads=3)), (RANGE, dict(batch=_batch(n_rows=1 << 30, max_rows=1 << 30)))]:
        assert cross(**kw) == code, (code, kw)


def test_calls_without_rows_do_nothing():
    """(Without a GPU a launch would fail.)"""
    none = _batch(n_rows=0, max_rows=0)
    assert append(batch=none) == 0 and read(batch=none) == 0 and kv4(batch=none) == 0 and cross(batch=none) == 0
    assert read(k=None, v=None) == 0


def test_calls_without_rows_need_no_buffers():
    none = _batch(n_rows=0, max_rows=0)
    assert append(batch=none, k=None, v=None, q=None, q_out=None) == 0
    assert read(batch=none, k=None, v=None) == 0
    assert kv4(batch=none, q=None, out=None) == 0
    assert cross(batch=none, q=None, out=None) == 0
    assert kv4(batch=none, q=A + 2) == ALIGN and append(batch=none, ks=100) == ALIGN


def test_structs_match_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "nfd.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name, struct in (("nfd_batch", N.NfdBatch), ("nfd_pages", N.NfdPages), ("nfd_rope", N.NfdRope), ("nfd_states", N.NfdStates)):
        body = re.findall(r"typedef struct \{([^{}]*)\} %s;" % name, text)[0]
        got = []
        for decl in filter(None, (d.strip() for d in body.split(";"))):
            kind = C.c_void_p if "*" in decl else {"int": C.c_int, "float": C.c_float, "long long": C.c_longlong}[
                re.match(r"(long long|int|float)", decl).group(1)]
            got += [(n.strip(), kind) for n in re.sub(r"^(const |unsigned |long long |int |float |char |void )+", "", decl)
                    .replace("*", "").split(",")]
        assert got == list(struct._fields_), name


def test_kv4_numbers_of_the_oracle():
    """The format's promises: every value is a bf16 number, no number is off by more than half a step unless it is clipped at
    the end of the range (then by less than a step), zero stays zero, and what is not finite is NaN."""
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 3, 64)) * np.exp(rng.uniform(-20, 20, (50, 3, 1)))).astype(np.float32)
    x[0, 0], x[1, 0, 3:9], x[2, 0, :32], x[3, 1, 5] = 0.0, 0.0, np.abs(x[2, 0, :32]), 1e30
    n, z, step = P.kv4_quantise(x)
    y = P.kv4_values(*P.kv4_bytes(n, z, step))
    f = y.astype(np.float32)
    assert np.array_equal(f, y) and not (f.view(np.uint32) & 0xFFFF).any()
    st = np.repeat(step, 32, -1)
    assert np.all(np.abs(y - x) <= st * 0.5000001 + (np.isin(n, (0, 15)) * 0.5 * st))
    assert np.all(y[x == 0] == 0) and np.all(z >= 0) and np.all(z <= 15)
    lo, hi = np.minimum(x.reshape(50, 3, 2, 32).min(-1), 0), np.maximum(x.reshape(50, 3, 2, 32).max(-1), 0)
    r = (hi - lo).astype(np.float64)
    assert np.all(15 * step >= r) and np.all(step <= np.maximum(r / 15 * 1.125, 2.0 ** -100))
    x[4, 0, 1], x[5, 1, 40], x[6, 2, :2] = np.nan, np.inf, (3e38, -3e38)
    n, z, step = P.kv4_quantise(x)
    bad = np.isnan(P.kv4_values(*P.kv4_bytes(n, z, step))).reshape(50, 3, 2, 32)
    assert bad[4, 0, 0].all() and bad[5, 1, 1].all() and bad[6, 2, 0].all() and bad.sum() == 96
