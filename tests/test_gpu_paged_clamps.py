"""Nonsense in device memory: no call reads or writes outside the rows that it was given."""
import pytest

from test_gpu_paged import _mods, _pool

pytestmark = pytest.mark.gpu

LOW = -(1 << 31)


@pytest.mark.parametrize("max_rows", [1, 8, 40, 200])
def test_row_starts_with_nonsense_in_them(max_rows):
    """Starts and ends below 0 and beyond the rows: they count as 0 and as n_rows.  All rows but the one sequence's that is left are as they were, and
    so is what lies around the buffers."""
    torch, N = _mods()
    i32 = lambda *x: torch.tensor(x, device="cuda", dtype=torch.int32)
    n, guard, heads, dh = 200, 2 * max_rows + 3, 2, 64
    m = min(3, max_rows)
    # sequences: n .. 4 (none), 4 .. -2^31 (none), -2^31 .. m (0 .. m), m .. -7 (none), and three below 0 (none)
    start = i32(1 << 30, 4, LOW, m, -7, LOW + 5, -1, LOW)
    n_seqs = start.numel() - 1
    lens = i32(*[n + 50] * n_seqs)
    table = torch.arange(n_seqs * 4, device="cuda", dtype=torch.int32).view(n_seqs, 4)
    b, good = (N.Batch(n, lens, table, row_start=x, max_rows=max_rows) for x in (start, i32(0, 0, 0, m, m, m, m, m)))
    pages = _pool("kv4", n_seqs * 4, heads, 64, dh, 1)
    pages.k_scale.fill_(0x3F87), pages.v_scale.fill_(0x3F87)
    gen = torch.Generator("cuda").manual_seed(0)
    for dt in (torch.bfloat16, torch.float32):
        big = torch.full((n + 2 * guard, heads, dh), float("nan"), device="cuda", dtype=dt)
        q = big[guard:guard + n]
        q.copy_(torch.randn(n, heads, dh, device="cuda", generator=gen))
        kv = torch.randn(n_seqs, 90, 2, heads, dh, device="cuda", generator=gen).to(dt)
        states = N.States(kv[:, :, 0], kv[:, :, 1])
        calls = [lambda bb, o: N.cross_attention(states, bb, q, o)]
        if dt == torch.bfloat16:
            calls.append(lambda bb, o: N.attention_kv4(pages, bb, q, o))
        for call in calls:
            outs = []
            for bb in (b, good):
                whole = torch.full((n + 2 * guard, heads * dh), 7.0, device="cuda", dtype=dt)
                call(bb, whole[guard:guard + n])
                outs.append(whole)
            assert torch.equal(outs[0], outs[1])
            rows = outs[0][guard:guard + m]
            assert rows.isfinite().all() and (rows != 7).any(1).all()
            outs[0][guard:guard + m] = 7.0
            assert (outs[0] == 7).all()
