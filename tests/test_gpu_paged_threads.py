"""The calls on the caller's own memory from several threads, and overlapped and replayed calls whose outputs were cleared before."""
import subprocess
import sys

import pytest

from test_gpu_paged import _one_of_each

pytestmark = pytest.mark.gpu

FIRST_CALLS = """
import threading
import torch
from paper_2506_01380_b200 import nfd as N
i32 = lambda *x: torch.tensor(x, device="cuda", dtype=torch.int32)
dev, n_threads = torch.device("cuda:0"), 8

def work(seed):
    # every kind of call, with rotations that differ from thread to thread
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *sh, dt=torch.bfloat16: torch.randn(sh, device="cuda", generator=g).to(dt)
    runs, outs = [], []
    for dh in (32, 64, 128):
        for rows in (1, 12, 140):
            pages, b = N.Pages.empty("kv4", 9, 2, 64, dh), N.Batch(rows, i32(500), torch.arange(9, device="cuda", dtype=torch.int32)[None])
            k, v, q, o = new(rows, 2, dh), new(rows, 2, dh), new(rows, 4, dh), new(rows, 4 * dh)
            qr, rope = torch.empty_like(q), N.Rope(dh, 0, 0, theta=1e4 + seed)
            ko = torch.zeros(rows, 2, dh, device="cuda")
            runs.append(lambda s, pages=pages, b=b, k=k, v=v, q=q, qr=qr, r=rope: N.kv_append(pages, b, k, v, r, q, qr, stream=s))
            runs.append(lambda s, pages=pages, b=b, ko=ko: N.pages_read(pages, b, ko, None, stream=s))
            runs.append(lambda s, pages=pages, b=b, q=qr, o=o: N.attention_kv4(pages, b, q, o, stream=s))
            outs += [qr, ko, o]
            for dt in (torch.bfloat16, torch.float32):
                st, qc, oc = N.States(new(1, 700, 2, dh, dt=dt), new(1, 700, 2, dh, dt=dt)), new(rows, 4, dh, dt=dt), new(rows, 4 * dh, dt=dt)
                runs.append(lambda s, st=st, b=N.Batch(rows, n_seqs=1), qc=qc, oc=oc: N.cross_attention(st, b, qc, oc, stream=s))
                outs.append(oc)
    return runs, outs

work_of = [work(i) for i in range(n_threads)]
streams = [torch.cuda.Stream() for _ in range(n_threads)]
torch.cuda.synchronize()
start, failed = threading.Barrier(n_threads), []

def body(i):
    try:
        torch.cuda.set_device(dev)
        start.wait()
        for run in work_of[i][0]:
            run(streams[i])
    except Exception as e:
        failed.append(repr(e))

threads = [threading.Thread(target=body, args=(i,)) for i in range(n_threads)]
for t in threads:
    t.start()
for t in threads:
    t.join()
torch.cuda.synchronize()
assert not failed, failed
first = [[o.clone() for o in outs] for _, outs in work_of]
for runs, outs in work_of:
    for o in outs:
        o.zero_()
    for run in runs:
        run(None)
torch.cuda.synchronize()
assert all(torch.equal(a, o) for f, (_, outs) in zip(first, work_of) for a, o in zip(f, outs))
print("same")
"""


def test_first_calls_from_several_threads():
    """In a process of its own: eight threads make every kernel's first call at once, each on a stream of its own."""
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=240)
    assert done.returncode == 0 and done.stdout.strip() == "same", done.stderr[-2000:]


def test_overlapping_calls_write_all_that_they_should():
    """Eager calls on two streams at once, several rounds, the outputs full of another number before each."""
    import torch
    calls = [c for c in _one_of_each(2)]
    for c in calls:
        c[1]()
    torch.cuda.synchronize()
    want = [[t.clone() for t in c[2]] for c in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for c in calls:
            if c[0] != "append":
                for t in c[2]:
                    t.fill_(7)
        torch.cuda.synchronize()
        for _ in range(3):
            for i, c in enumerate(calls):
                if c[0] != "append":
                    c[1](streams[i % 2])
        torch.cuda.synchronize()
        for c, f in zip(calls, want):
            assert all(torch.equal(a, b) for a, b in zip(c[2], f)), c[0]


@pytest.mark.parametrize("rows", [1, 12, 150])
def test_replays_go_by_what_device_memory_holds_then(rows):
    """A step of all calls captured once and replayed with other lengths, tables, row starts, rows and masks in place, the outputs full of
    another number: bit for bit what eager calls write with these."""
    import torch
    from paper_2506_01380_b200 import nfd as N
    g = torch.Generator("cuda").manual_seed(rows)
    i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)
    new = lambda *sh, dt=torch.bfloat16: torch.randn(sh, device="cuda", generator=g).to(dt)
    n = 2 * rows + 1
    x, enc = new(n, 4 + 2 * 2, 64), new(2, 300, 2, 2, 64)
    lens, keys, table, start = i32([rows, rows]), i32([300, 20]), i32([[0, 1, 2, 3, 4], [5, 6, 7, 8, 9]]), i32([0, rows, 2 * rows])
    mask = torch.rand(2, 300, device="cuda", generator=g) < 0.5
    b = N.Batch(n, lens, table, row_start=start, max_rows=rows)
    c = N.Batch(n, keys, row_start=start, max_rows=rows)
    rope = N.Rope(16, 24, 24, frame_tokens=12, grid_w=4)
    history = new(2, 300, 2, 64)

    def outputs():
        full = lambda *sh, dt=torch.bfloat16: torch.full(sh, 7.0, device="cuda", dtype=dt)
        pages = N.Pages.empty("kv4", 10, 2, 64, 64)
        own = N.Pages.empty(torch.bfloat16, 10, 2, 64, 64)
        for t in (pages, own):                                         # what lies in the pages before the step
            N.kv_append(t, N.Batch(600, i32([300, 300]), i32([[0, 1, 2, 3, 4], [5, 6, 7, 8, 9]])), history.view(600, 2, 64), history.view(600, 2, 64))
        return dict(pages=pages, own=own, q=full(n, 4, 64), k=full(n, 2, 64, dt=torch.float32), v=full(n, 2, 64), o=full(n, 256), c=full(n, 256),
                    f=full(n, 256, dt=torch.float32))

    def step(s):
        q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
        N.kv_append(s["pages"], b, k, v, rope, q, s["q"])
        N.kv_append(s["own"], b, k, v, rope)
        N.pages_read(s["pages"], b, s["k"], None)
        N.pages_read(s["own"], b, None, s["v"])
        N.attention_kv4(s["pages"], b, x[:, :4], s["o"], frame_tokens=12, window=5)
        N.cross_attention(N.States(enc[:, :, 0], enc[:, :, 1], mask), c, x[:, :4], s["c"])
        N.cross_attention(N.States(wide[:, :, 0], wide[:, :, 1], mask), c, xf, s["f"])

    wide, xf = enc.float(), x[:, :4].float()
    held = lambda s: [s["pages"].k, s["pages"].v, s["pages"].k_scale, s["pages"].v_scale, s["own"].k, s["own"].v] + [s[a] for a in "qkvocf"]
    s = outputs()
    step(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s)
    # (the last row stays behind the last sequence; pages of the two sequences change places, one entry is no page)
    for lengths, order, starts in (([290, 77 + rows], [[9, 8, 7, 6, 5], [0, 3, 1, 2, 4]], [0, rows - 1, 2 * rows - 1]),
                                   ([rows // 2, 10000], [[3, 1, 2, 8, 6], [0, -1, 9, 7, 5]], [1, rows, 2 * rows])):
        lens.copy_(i32(lengths)), table.copy_(i32(order)), start.copy_(i32(starts)), keys.copy_(keys.flip(0))
        x.copy_(x.flip(0)), xf.copy_(x[:, :4]), mask.logical_not_()
        fresh, again = outputs(), outputs()
        for a, f in zip(held(s), held(fresh)):
            a.copy_(f)
        graph.replay()
        step(again)
        torch.cuda.synchronize()
        for i, (a, f) in enumerate(zip(held(s), held(again))):
            assert torch.equal(a, f), (lengths, i)
        assert all((s[a][2 * rows:] == 7).all() for a in "qkvocf") and (s["c"] != 7).any() and (s["o"] != 7).any()
