"""Arguments that the calls around a block's projections do not look at, whatever they are.  No GPU: batches without rows, whose other arguments are
checked all the same."""
from tests.test_block_refusals import _mod, _norm, norm, packed, pages, rotate
from tests.test_paged_refusals import A, ALIGN, RANGE, _batch

NOWHERE = A + 1                                            # aligned to nothing


def test_gate_norm_without_y_looks_at_no_gate_and_without_h_at_no_scale_and_shift():
    assert norm(n=0, mod=_mod(gate=NOWHERE)) == norm(n=0, mod=_mod(scale=NOWHERE)) == norm(n=0, mod=_mod(shift=NOWHERE)) == ALIGN
    assert norm(n=0, mod=_mod(stride=8)) == RANGE
    assert norm(n=0, y=None, mod=_mod(gate=NOWHERE), xo=NOWHERE, xos=-5, post=_norm(kind=9, weight=NOWHERE)) == 0
    assert norm(n=0, y=None, mod=_mod(gate=NOWHERE, scale=None, shift=None, stride=-3)) == 0
    assert norm(n=0, h=None, mod=_mod(scale=NOWHERE, shift=NOWHERE), pre=_norm(kind=9, bias=NOWHERE)) == 0
    assert norm(n=0, y=None, mod=_mod(gate=NOWHERE, scale=NOWHERE)) == norm(n=0, h=None, mod=_mod(gate=NOWHERE)) == ALIGN


def test_packed_prompts_look_at_no_lengths_and_no_table():
    none = dict(n_rows=0, max_rows=0)
    assert packed(batch=_batch(kv_len=NOWHERE, table=NOWHERE, table_len=-7, **none)) == 0
    assert packed(batch=_batch(row_start=NOWHERE, **none)) == ALIGN
    assert pages(batch=_batch(kv_len=NOWHERE, **none)) == pages(batch=_batch(table=NOWHERE, **none)) == ALIGN


def test_rotation_without_heads_looks_at_no_rows():
    assert rotate(n=0, h2=0, y=NOWHERE, ys=-1, yo=NOWHERE, yos=-2) == rotate(n=0, h=0, x=NOWHERE, xs=-1, xo=NOWHERE, xos=-2) == 0
    assert rotate(n=0, y=NOWHERE) == ALIGN
