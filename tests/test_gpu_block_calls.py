"""The calls around a block's projections as a program may make them: first calls inside a capture and from several threads, no rows,
strides and sizes far out, the same call again and again."""
import subprocess
import sys

import numpy as np
import pytest

from test_gpu_block import EVER, _batch, _check_norm, _check_pages, _check_rotate, _int, _mods

pytestmark = pytest.mark.gpu

ONE_OF_EACH = """
import threading
import torch
from paper_2506_01380_b200 import nfd as N
i32 = lambda *x: torch.tensor(x, device="cuda", dtype=torch.int32)

def work(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *sh, dt=torch.bfloat16: torch.randn(sh, device="cuda", generator=g).to(dt)
    runs, outs = [], []
    for dt in (torch.bfloat16, torch.float32):
        for dh in (32, 64, 128):
            for rows in (1, 12, 140, 400):
                b = N.Batch(rows, i32(500), table=torch.arange(18, device="cuda", dtype=torch.int32)[None])
                q, o, op = new(rows, 4, dh, dt=dt), new(rows, 4 * dh, dt=dt), new(rows, 4 * dh, dt=dt)
                k, v = new(rows, 2, dh, dt=dt), new(rows, 2, dh, dt=dt)
                for page in (32, 30):
                    pages = N.Pages(new(18, 2, page, dh, dt=dt), new(18, 2, page, dh, dt=dt))
                    out = new(rows, 4 * dh, dt=dt)
                    runs.append(lambda s, pages=pages, b=b, q=q, out=out: N.attention_pages(pages, b, q, out, stream=s))
                    outs.append(out)
                runs.append(lambda s, b=N.Batch(rows, n_seqs=1), q=q, k=k, v=v, op=op: N.attention_packed(b, q, k, v, op, stream=s))
                r, pos = N.Rope(dh, 0, 0, theta=1e4 + seed), torch.arange(3 * rows, device="cuda").view(rows, 3).int()
                qo, ko = new(rows, 4, dh, dt=dt), new(rows, 2, dh, dt=dt)
                for hv in (False, True):
                    runs.append(lambda s, r=r, pos=pos, q=q, qo=qo, k=k, ko=ko, hv=hv: N.rotate(r, pos, q, qo, k, ko, halves=hv, stream=s))
                outs += [op, qo, ko]
        for n, width in ((5, 128), (40, 1024), (3000, 1024), (1300, 8192)):
            x, y, xo, h = new(n, width), new(n, width, dt=dt), new(n, width), new(n, width, dt=dt)
            runs.append(lambda s, x=x, y=y, xo=xo, h=h: N.gate_norm(x, y, xo, h, pre=N.Norm("layer"), post=N.Norm("rms"), stream=s))
            outs += [xo, h]
    return runs, outs
"""

CAPTURED = ONE_OF_EACH + """
runs, outs = work(0)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):                      # the first calls of this process
    for run in runs:
        run(None)
for o in outs:
    o.fill_(7.0)
graph.replay()
got = [o.clone() for o in outs]
for run in runs:
    run(None)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, outs))
"""

THREADS = ONE_OF_EACH + """
n = 6
work_of = [work(i) for i in range(n)]
streams = [torch.cuda.Stream() for _ in range(n)]
torch.cuda.synchronize()
start, failed = threading.Barrier(n), []

def body(i):
    try:
        torch.cuda.set_device(0)
        start.wait()
        for run in work_of[i][0]:
            run(streams[i])
    except Exception as e:
        failed.append(repr(e))

threads = [threading.Thread(target=body, args=(i,)) for i in range(n)]
for t in threads:
    t.start()
for t in threads:
    t.join()
torch.cuda.synchronize()
assert not failed, failed
first = [[o.clone() for o in outs] for _, outs in work_of]
for runs, outs in work_of:                         # and again, one after the other
    for o in outs:
        o.fill_(7.0)
    for run in runs:
        run(None)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for f, (_, outs) in zip(first, work_of) for a, b in zip(f, outs))
"""


@pytest.mark.parametrize("program", [CAPTURED, THREADS], ids=["captured", "threads"])
def test_first_calls(program):
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_a_step_without_rows():
    """A batch of no rows: empty tensors, which have no address."""
    torch, N = _mods()
    new = lambda *sh: torch.zeros(sh, device="cuda", dtype=torch.bfloat16)
    b = N.Batch(0, _int([5, 9]), _int(np.zeros((2, 1))))
    assert N.attention_pages(N.Pages(new(1, 2, 16, 64), new(1, 2, 16, 64)), b, new(0, 4, 64), new(0, 256)).numel() == 0
    assert N.attention_packed(N.Batch(0, row_start=_int([0, 0, 0])), new(0, 4, 64), new(0, 2, 64), new(0, 2, 64), new(0, 256)).numel() == 0
    N.rotate(N.Rope(64, 0, 0), torch.zeros(0, 3, device="cuda", dtype=torch.int32), new(0, 4, 64), x2=new(0, 2, 64))
    N.gate_norm(new(0, 64), new(0, 64), h=new(0, 64), pre=N.Norm("rms"))
    N.attention_packed(N.Batch(7, row_start=_int([0, 0, 0]), max_rows=5), new(7, 4, 64), new(7, 2, 64), new(7, 2, 64), new(7, 256))     # rows of nobody
    torch.cuda.synchronize()


@pytest.mark.parametrize("dh", [64, 128])
def test_fewer_rows_than_a_block_has_keys(dh):
    """Tensors smaller than the boxes that are copied."""
    torch, N = _mods()
    for rows in (9, 50):
        q, k, v = (torch.randn(rows, h, dh, device="cuda").bfloat16() for h in (32, 1, 1))
        out = torch.zeros(rows, 32 * dh, device="cuda", dtype=torch.bfloat16)
        N.attention_packed(N.Batch(rows, n_seqs=1), q, k, v, out)
        s = torch.einsum("ihd,jgd->hij", q.double(), k.double()) / dh ** 0.5
        s.masked_fill_(torch.ones(rows, rows, device="cuda").triu(1).bool(), -torch.inf)
        want = torch.einsum("hij,jgd->ihd", s.softmax(-1), v.double()).reshape(rows, -1)
        # (P's rounding and the result's, half a step of bf16 each of at most the largest value, and as much again for exponentials and sums)
        assert (out.double() - want).abs().max() <= 4 * 2.0 ** -8 * v.abs().max()


def test_rows_far_apart():
    """Strides that take the rows beyond 2^32 bytes."""
    torch, N = _mods()
    n, wide = 70000, 1 << 15
    x = torch.empty(n, wide, device="cuda", dtype=torch.bfloat16)
    q, k, v = (x[:, a:a + 128].unflatten(1, (2, 64)) for a in (0, 1000 * 8, wide - 128))
    for t in (q, k, v):
        t.copy_(torch.randn(n, 2, 64, device="cuda"))
    rows = [300, 69000, 40, 600]
    start = _int(np.concatenate([[0], np.cumsum(rows)]))
    b = N.Batch(n, row_start=start, max_rows=69000)
    o1, o2 = (torch.zeros(n, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    N.attention_packed(b, q, k, v, o1, window=500)
    N.attention_packed(b, q.contiguous(), k.contiguous(), v.contiguous(), o2, window=500)
    assert torch.equal(o1, o2) and o1[69900:69940].abs().sum() > 0
    pos = torch.arange(3 * n, device="cuda").view(n, 3).int()
    r = N.Rope(16, 24, 24)
    a, c = q.contiguous(), k.contiguous()
    N.rotate(r, pos, a, x2=c)
    N.rotate(r, pos, q, x2=k)
    assert torch.equal(a, q) and torch.equal(c, k)
    h = torch.zeros(n, 64, device="cuda", dtype=torch.bfloat16)
    N.gate_norm(x[:, 8:72], x[:, 4096:4160], x[:, 256:320], h, pre=N.Norm("rms"))
    xo, h2 = N.gate_norm(x[:, 8:72].contiguous(), x[:, 4096:4160].contiguous(), torch.zeros_like(h), torch.zeros_like(h), pre=N.Norm("rms"))
    assert torch.equal(h, h2) and torch.equal(xo, x[:, 256:320])


@pytest.mark.parametrize("page", [8, 16, 24, 96, 128, 200, 30])
def test_pages_of_every_kind_of_box(page):
    for dh in (64, 128):
        for rows in (100, 400):
            _check_pages("bfloat16", [rows, rows // 3], [1500, 700], 6, 3, dh, page, 1500 // page + 1, 1, 600, seed=page)
            _check_pages("bfloat16", [rows], [1500], 2, 1, dh, page, 1500 // page + 1, 77, 3, seed=page)


@pytest.mark.parametrize("seqs", [2, 33, 128, 130])
@pytest.mark.parametrize("rows", [3, 90])
def test_sequences_of_any_length_in_any_order(seqs, rows):
    """What is dealt out longest first reaches every row, with row starts and without, sequences without rows or tokens among them."""
    torch, N = _mods()
    rng = np.random.default_rng(seqs + rows)
    lens = rng.integers(0, 700, seqs)
    lens[rng.integers(0, seqs, seqs // 3)] = 650
    n = rng.integers(0, rows + 1, seqs)
    n[0] = rows
    _check_pages("bfloat16", list(n), list(lens), 4, 2, 64, 32, 22, 1, EVER, seed=seqs, extra=5)
    _check_pages("bfloat16", list(n), list(lens), 4, 2, 128, 32, 10, 50, 2, seed=seqs, extra=5, max_rows=rows - 1)
    g = torch.Generator("cuda").manual_seed(rows)
    pages = N.Pages(*(torch.randn(22 * seqs, 2, 32, 64, device="cuda", generator=g).bfloat16() for _ in range(2)))
    q = torch.randn(seqs * rows, 4, 64, device="cuda", generator=g).bfloat16()
    table, held = torch.randperm(22 * seqs, device="cuda").int().view(seqs, 22), _int(lens)
    outs = [torch.full((seqs * rows, 256), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    N.attention_pages(pages, N.Batch(seqs * rows, held, table=table), q, outs[0])
    N.attention_pages(pages, N.Batch(seqs * rows, held, table=table, row_start=_int(np.arange(seqs + 1) * rows), max_rows=rows), q, outs[1])
    assert torch.equal(*outs)


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_the_same_call_again(dh):
    """Tiles that begin and end in other blocks, groups in turn, pieces: the same bits whenever it runs."""
    torch, N = _mods()
    g = torch.Generator("cuda").manual_seed(dh)
    for rows, frame, window in (([1232] * 3, 77, 3), ([1000, 30, 700], 1, 100), ([130] * 9, 1, EVER), ([3000], 1, EVER), ([250, 380, 100], 336, 1)):
        b, n, _ = _batch(rows)
        q, k, v = (torch.randn(n, m, dh, device="cuda", generator=g).bfloat16() for m in (4, 4, 4))
        outs = [torch.zeros(n, 4 * dh, device="cuda", dtype=torch.bfloat16) for _ in range(12)]
        for o in outs:
            N.attention_packed(b, q, k, v, o, frame_tokens=frame, window=window)
        assert all(torch.equal(o, outs[0]) for o in outs)
    pages = N.Pages(*(torch.randn(300, 2, 32, dh, device="cuda", generator=g).bfloat16() for _ in range(2)))
    for rows, length in ((100, 9000), (400, 9000), (1, 9000), (900, 3000)):
        b = N.Batch(rows, _int([length]), torch.randperm(300, device="cuda").int()[None].contiguous())
        q = torch.randn(rows, 8, dh, device="cuda", generator=g).bfloat16()
        outs = [torch.zeros(rows, 8 * dh, device="cuda", dtype=torch.bfloat16) for _ in range(12)]
        for o in outs:
            N.attention_pages(pages, b, q, o)
        assert all(torch.equal(o, outs[0]) for o in outs)


def test_rotate_more_places_than_threads():
    _check_rotate("bfloat16", 300, 40, 8, 128, (32, 48, 48), False, False)
    _check_rotate("float32", 20, 100, 30, 64, (0, 32, 32), True, True, in_place=True)


@pytest.mark.parametrize("xt,dt", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "bfloat16")])
def test_gate_norm_many_wide_rows(xt, dt):
    for width in (4104, 8200, 16384):
        _check_norm(xt, dt, 1300, width, "layer", True, True, True, True, True, in_place=width == 8200)
        _check_norm(xt, dt, 1300, width, "rms", False, True, False, True, False, use_h=False)
        _check_norm(xt, dt, 1300, width, "rms", False, False, True, True, False, use_y=False)


@pytest.mark.parametrize("xt,dt", [("float32", "float32"), ("float32", "bfloat16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
def test_gate_norm_any_width(xt, dt):
    """Few rows and many: other plans, the same sums in the same order."""
    torch, N = _mods()
    x, y = torch.randn(1300, 16384, device="cuda").to(getattr(torch, xt)), torch.randn(1300, 16384, device="cuda").to(getattr(torch, dt))
    for width in [*range(8, 640, 8), *range(640, 16385, 328), 4096, 8192, 16384]:
        got = [N.gate_norm(x[a:b, :width], y[a:b, :width], torch.empty(b - a, width, device="cuda", dtype=x.dtype), pre=N.Norm("layer"),
                           post=N.Norm("rms"), h=torch.empty(b - a, width, device="cuda", dtype=y.dtype))
               for a, b in ((0, 1300), (0, 200), (1200, 1300))]
        for k in (0, 1):
            assert torch.equal(got[0][k][:200], got[1][k]) and torch.equal(got[0][k][1200:], got[2][k]), width


def test_python_refuses():
    torch, N = _mods()
    new = lambda *sh, dt=torch.bfloat16: torch.zeros(sh, device="cuda", dtype=dt)
    b = N.Batch(4, _int([9]), _int([[0]]))
    bf, kv4 = N.Pages(new(1, 2, 16, 64), new(1, 2, 16, 64)), N.Pages.empty("kv4", 1, 2, 16, 64)
    q, out = new(4, 4, 64), new(4, 256)
    for bad in (lambda: N.attention_pages(kv4, b, q, out), lambda: N.attention_pages(bf, b, q.float(), out),
                lambda: N.attention_pages(bf, b, q, new(4, 128)), lambda: N.attention_pages(bf, b, new(5, 4, 64), out),
                lambda: N.attention_pages(bf, b, new(4, 8, 64)[:, ::2], out),
                lambda: N.attention_packed(b, q, new(4, 2, 64, dt=torch.float32), new(4, 2, 64), out),
                lambda: N.attention_packed(b, q, new(4, 2, 64), new(3, 2, 64), out),
                lambda: N.attention_packed(b, q.cpu(), new(4, 2, 64), new(4, 2, 64), out),
                lambda: N.rotate(N.Rope(64, 0, 0), new(4, 3), q), lambda: N.rotate(N.Rope(64, 0, 0), new(4, 2, dt=torch.int32), q),
                lambda: N.gate_norm(new(4, 64), h=new(4, 64)), lambda: N.gate_norm(new(4, 64), new(4, 32)), lambda: N.gate_norm(new(4, 64)),
                lambda: N.gate_norm(new(4, 64), h=new(4, 64), pre=N.Norm("rms", weight=new(32))),
                lambda: N.Modulation(gate=new(2, 64)), lambda: N.Modulation(gate=new(2, 64), scale=new(2, 64, dt=torch.float32), rows_per_mod=2)):
        with pytest.raises(AssertionError):
            bad()
    for code, bad in ((-4, lambda: N.attention_pages(bf, b, new(4, 3, 64), new(4, 192))),
                      (-4, lambda: N.attention_pages(bf, b, q, out, frame_tokens=0)),
                      (-1, lambda: N.rotate(N.Rope(32, 0, 0), new(4, 3, dt=torch.int32), q)),
                      (-4, lambda: N.gate_norm(new(4, 12), h=new(4, 12), pre=N.Norm("rms")))):
        with pytest.raises(N.NfdError) as e:
            bad()
        assert e.value.code == code
