"""rtprune_page_map refuses outputs that lie over its inputs or one another, before anything is launched (no GPU needed)."""
import pytest

from paper_2605_00392_b200 import binding

INVALID = 1
P = 1 << 20            # addresses that are never followed: every call here returns before a launch
BATCH, ROWS, FREE, STRIDE, PAGES = 3, 10, 7, 6, 4
INPUTS = dict(offsets=BATCH + 1, ctx=BATCH, index=ROWS, base=BATCH, free=FREE, head=1)
OUTPUTS = dict(slots=ROWS, pos=ROWS, lens=BATCH, state=2)


def _map(**kw):
    a = dict(offsets=P, ctx=2 * P, batch=BATCH, rows=ROWS, index=3 * P, base=4 * P, free=5 * P, head=6 * P, n_free=FREE, page=16, table=7 * P,
             stride=STRIDE, pages=PAGES, slots=8 * P, pos=9 * P, lens=10 * P, state=11 * P)
    at = dict(a)
    a.update({k: v(at) if callable(v) else v for k, v in kw.items()})
    return binding.lib().rtprune_page_map(None, *a.values())


@pytest.mark.parametrize("out", OUTPUTS)
@pytest.mark.parametrize("other", [*INPUTS, *OUTPUTS])
def test_outputs_over_other_memory(out, other):
    if out == other:
        return
    words = {**INPUTS, **OUTPUTS}
    # the same address; the last word of one the first of the other
    assert _map(**{out: lambda a: a[other]}) == INVALID
    assert _map(**{out: lambda a: a[other] + 4 * (words[other] - 1)}) == INVALID
    assert _map(**{out: lambda a: a[other] - 4 * (words[out] - 1)}) == INVALID


@pytest.mark.parametrize("other", [*INPUTS, *OUTPUTS])
def test_tables_over_other_memory(other):
    words = {**INPUTS, **OUTPUTS}[other]
    for row in range(BATCH):
        for word in (0, PAGES - 1):
            at = 7 * P + 4 * (row * STRIDE + word)
            assert _map(**{other: at}) == INVALID, (row, word)
            assert _map(**{other: at - 4 * (words - 1)}) == INVALID, (row, word)
    if words > STRIDE - PAGES:                     # begins in the gap behind a row's entries and reaches the next one's
        assert _map(**{other: 7 * P + 4 * PAGES}) == INVALID
