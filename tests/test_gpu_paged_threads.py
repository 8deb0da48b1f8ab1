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
