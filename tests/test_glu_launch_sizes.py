"""Sizes at the end of what a launch of the gated feed-forward holds (CPU): the form
that is taken can be launched wherever any can, and where none can the call is
refused by its sizes."""
import random

import pytest

from paper_2606_01143_amd import binding as B
from test_glu_rule import forms

MOST = 2 ** 32 - 1  # threads of a launch
# rows and result columns of a form's tile, threads of its workgroup, in the rule's order
FWD = [(64, 64, 256), (128, 64, 256), (128, 64, 256), (192, 128, 512), (256, 128, 512), (32, 32, 256)]
BWD = [(64, 128, 256), (128, 128, 256), (128, 128, 256), (192, 256, 512), (256, 256, 512), (32, 64, 192), (32, 32, 256)]


def threads(form, experts, rows, columns):
    """Of a launch: at most one tile of rows that is not whole for every expert that
    has any, workgroups a multiple of the eight XCDs."""
    high, wide, of_group = form
    some = min(experts, rows)
    groups = -(-columns // wide) * ((rows + some * (high - 1)) // high)
    return -(-groups // 8) * 8 * of_group


def accepted(e, rows, i, o):
    """The sizes that every product of rows by expert takes."""
    return ((rows // 32 + e) * (2 * (max(i, o) // 32 + 1)) < 2 ** 31
            and e * 2 * (i // 32 + 1) * (o // 32 + 1) < 2 ** 31)


def _sizes():
    rng = random.Random(5)
    # 60 experts of 16M columns: the 64-row tiles do not fit, larger ones do
    out = [(60, 384, 8, 1 << 24), (1, 64, 8, 1 << 30), (30, 30, 16, 1 << 25), (1, 2147482623, 8, 8), (1024, 1 << 30, 8, 8)]
    while len(out) < 3000:
        e = rng.choice([1, 1, 2, 8, 60, 128, 1024])
        rows = int(2 ** rng.uniform(0, 31)) - 1
        mid, other = (max(8, int(2 ** rng.uniform(3, 31)) // 8 * 8) for _ in range(2))
        if 0 < rows <= 2147482623 and max(mid, other) <= 2147482616 and accepted(e, rows, mid, other):
            if rows / 64 * mid / 64 > 1 << 20 or e * mid / 64 > 1 << 20:  # near the end
                out.append((e, rows, other, mid))
    return out


def test_the_form_can_be_launched():
    sizes = _sizes()
    some = [0, 0]
    for (e, rows, other, mid), taken in zip(sizes, forms(sizes)):
        for k, (table, form) in enumerate(zip((FWD, BWD), taken)):
            fits = [threads(f, e, rows, mid) <= MOST for f in table]
            if any(fits):
                assert fits[form], (e, rows, other, mid, k, form)
                some[k] += not all(fits)
    assert min(some) >= 5  # sizes where only some forms fit


def _at(i):
    return 0x100000000000 + i * (1 << 41)


def _glu(e, rows, other, mid):
    fwd = (0, e, rows, other, mid, _at(1), _at(2), rows, None, _at(3), _at(4), _at(5), None, None, None, None, None)
    bwd = (0, e, rows, mid, other, _at(1), _at(2), _at(3), _at(4), None, _at(5), None, _at(6), _at(7), _at(8), None)
    return ("spr_glu_fwd", fwd, FWD), ("spr_glu_bwd", bwd, BWD)


@pytest.mark.parametrize("e,rows,other,mid", [(128, 128, 8, 1 << 23), (1, 1, 8, 2147482616), (1024, 2147482000, 8, 8)])
def test_what_no_launch_holds_is_refused(e, rows, other, mid):
    """(The addresses are never dereferenced: nothing is launched.)"""
    assert accepted(e, rows, other, mid)
    refused = 0
    for name, args, table in _glu(e, rows, other, mid):
        if any(threads(f, e, rows, mid) <= MOST for f in table):
            continue
        refused += 1
        assert B.STATUS[getattr(B.lib(), name)(*args)] == "SPR_ERR_INVALID_ARG", name
        assert "launch" in B.last_error(), B.last_error()
    assert refused
