"""Refusals of the experts' calls (CPU): sizes, types, alignment, overlaps,
pairs and workspaces, before anything is launched.  The addresses are never
dereferenced."""
import pytest
import torch

from paper_2606_01143_amd import binding as B


def _at(i, off=0):
    return 0x7F0000000000 + i * (1 << 34) + off


def _call(name, base, **kw):
    a = dict(base)
    a.update(kw)
    return B.STATUS[getattr(B.lib(), name)(*a.values(), None)]


PLAN = dict(E=16, k=2, T=10, experts=_at(1), offsets=_at(2), row_token=_at(3), pos=_at(4), ws=_at(5), wsb=1 << 20)
FWD = dict(E=4, rows=10, i=64, o=32, offsets=_at(1), x=_at(2), x_rows=10, row_token=None, w=_at(3), y=_at(4), w2=_at(5),
           y2=_at(6))
BWD_X = dict(E=4, rows=10, i=64, o=32, offsets=_at(1), dy=_at(2), w=_at(3), dy2=_at(4), w2=_at(5), dx=_at(6))
BWD_W = dict(E=4, rows=10, i=64, o=32, offsets=_at(1), x=_at(2), x_rows=10, row_token=None, dy=_at(3), dw=_at(4),
             dy2=_at(5), dw2=_at(6), overwrite=1)
COMBINE = dict(T=10, k=2, rows=20, w=64, y=_at(1), pos=_at(2), weights=_at(3), add=_at(4), out=_at(5))
COMBINE_BWD = dict(T=10, k=2, rows=20, w=64, dout=_at(1), y=_at(2), pos=_at(3), weights=_at(4), dy=_at(5), dw=_at(6))


@pytest.mark.parametrize("kw,status", [
    (dict(E=0), "UNSUPPORTED"), (dict(E=1025), "UNSUPPORTED"), (dict(k=0), "INVALID_ARG"), (dict(k=17), "INVALID_ARG"),
    (dict(T=-1), "INVALID_ARG"), (dict(T=2147483647), "INVALID_ARG"), (dict(experts=None), "INVALID_ARG"),
    (dict(offsets=None), "INVALID_ARG"), (dict(pos=_at(4, 2)), "MISALIGNED"), (dict(pos=_at(1)), "ALIASING"),
    (dict(row_token=_at(4, 8)), "ALIASING"),
    # more than 4096 choices: the plan needs its workspace
    (dict(T=40000, ws=None), "WORKSPACE"), (dict(T=40000, wsb=4), "WORKSPACE"),
    (dict(T=40000, ws=_at(5, 4)), "MISALIGNED"), (dict(T=40000, ws=_at(2)), "ALIASING")])
def test_plan(kw, status):
    assert _call("spr_experts_plan", PLAN, **kw) == "SPR_ERR_" + status
    assert B.last_error()


SIZES = [(dict(E=0), "UNSUPPORTED"), (dict(E=2000), "UNSUPPORTED"), (dict(rows=-1), "INVALID_ARG"),
         (dict(i=12), "UNSUPPORTED"), (dict(o=0), "UNSUPPORTED"), (dict(o=4), "UNSUPPORTED"),
         (dict(offsets=None), "INVALID_ARG"), (dict(offsets=_at(1, 1)), "MISALIGNED"),
         (dict(rows=2147483647, i=1 << 20, x_rows=2147483647), "INVALID_ARG"),
         (dict(E=1024, i=1 << 20, o=1 << 20), "INVALID_ARG")]


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(x_rows=9), "INVALID_ARG"), (dict(x_rows=0, row_token=_at(7)), "INVALID_ARG"),
    (dict(row_token=_at(7, 2)), "MISALIGNED"), (dict(w2=None), "INVALID_ARG"), (dict(y2=None), "INVALID_ARG"),
    (dict(x=None), "INVALID_ARG"), (dict(y=None), "INVALID_ARG"), (dict(w=_at(3, 8)), "MISALIGNED"),
    (dict(y=_at(2)), "ALIASING"), (dict(y2=_at(4)), "ALIASING"), (dict(y=_at(5)), "ALIASING"),
    (dict(y=_at(1)), "ALIASING")])
def test_fwd(kw, status):
    assert _call("spr_experts_fwd", FWD, **kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", [(a, b) for a, b in
                                       [({k: v for k, v in kw.items() if k != "x_rows"}, s) for kw, s in SIZES]] + [
    (dict(w2=None), "INVALID_ARG"), (dict(dy2=None), "INVALID_ARG"), (dict(dx=None), "INVALID_ARG"),
    (dict(dx=_at(2)), "ALIASING"), (dict(dx=_at(5, 64)), "ALIASING"), (dict(dy=_at(2, 4)), "MISALIGNED")])
def test_bwd_x(kw, status):
    assert _call("spr_experts_bwd_x", BWD_X, **kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", SIZES + [
    (dict(x_rows=9), "INVALID_ARG"), (dict(dy2=None), "INVALID_ARG"), (dict(dw2=None), "INVALID_ARG"),
    (dict(dw=None), "INVALID_ARG"), (dict(dw=_at(4, 8)), "MISALIGNED"), (dict(dw2=_at(4, 4096)), "ALIASING"),
    (dict(dw=_at(3)), "ALIASING"), (dict(dw=_at(2)), "ALIASING"), (dict(x=None), "INVALID_ARG")])
def test_bwd_w(kw, status):
    assert _call("spr_experts_bwd_w", BWD_W, **kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "INVALID_ARG"), (dict(k=0), "INVALID_ARG"), (dict(rows=-1), "INVALID_ARG"), (dict(w=12), "UNSUPPORTED"),
    (dict(T=1 << 30), "INVALID_ARG"), (dict(pos=None), "INVALID_ARG"), (dict(out=None), "INVALID_ARG"),
    (dict(y=_at(1, 8)), "MISALIGNED"), (dict(out=_at(1)), "ALIASING"), (dict(out=_at(4, 16)), "ALIASING"),
    (dict(out=_at(3)), "ALIASING")])
def test_combine(kw, status):
    assert _call("spr_experts_combine_fwd", COMBINE, **kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), "INVALID_ARG"), (dict(k=0), "INVALID_ARG"), (dict(w=4), "UNSUPPORTED"), (dict(y=None), "INVALID_ARG"),
    (dict(dw=None), "INVALID_ARG"), (dict(dout=None), "INVALID_ARG"), (dict(dy=_at(2)), "ALIASING"),
    (dict(dy=_at(1)), "ALIASING"), (dict(dw=_at(4)), "ALIASING"), (dict(dw=_at(6, 1)), "MISALIGNED")])
def test_combine_bwd(kw, status):
    assert _call("spr_experts_combine_bwd", COMBINE_BWD, **kw) == "SPR_ERR_" + status


def test_nothing_to_do_launches_nothing():
    """No rows or tokens: the shapes are checked, the pointers are not needed."""
    assert _call("spr_experts_fwd", FWD, rows=0, x=None, y=None, w2=None, y2=None) == "SPR_OK"
    assert _call("spr_experts_bwd_x", BWD_X, rows=0, dy=None, dx=None) == "SPR_OK"
    assert _call("spr_experts_bwd_w", BWD_W, rows=0, overwrite=0) == "SPR_OK"
    assert _call("spr_experts_combine_fwd", COMBINE, T=0) == "SPR_OK"
    assert _call("spr_experts_combine_bwd", COMBINE_BWD, T=0) == "SPR_OK"


def test_no_rows_of_a_pair():
    """An empty tensor's pointer is NULL: no half of a pair is missing."""
    assert _call("spr_experts_fwd", FWD, rows=0, x=None, y=None, y2=None) == "SPR_OK"
    assert _call("spr_experts_bwd_x", BWD_X, rows=0, dy=None, dy2=None, dx=None) == "SPR_OK"
    assert _call("spr_experts_bwd_w", BWD_W, rows=0, x=None, dy=None, dy2=None, overwrite=0) == "SPR_OK"


def test_plan_workspace_size():
    assert B.experts_plan_workspace_size(8, 2, 2048) == 0
    mid, large = B.experts_plan_workspace_size(8, 2, 2049), B.experts_plan_workspace_size(1024, 8, 1 << 20)
    assert 0 < mid < large <= 1 << 20
    with pytest.raises(B.SprError):
        B.experts_plan_workspace_size(8, 9, 4)


def test_binding_types_and_shapes():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    off, x, w, y = i32(5), bf(10, 16), bf(4, 16, 24), bf(10, 24)
    with pytest.raises(ValueError, match="x: torch.float16"):
        B.experts_fwd(off, x.half(), w, y)
    with pytest.raises(ValueError, match="offsets: torch.int64"):
        B.experts_fwd(off.long(), x, w, y)
    with pytest.raises(ValueError, match="offsets: shape"):
        B.experts_fwd(i32(4), x, w, y)
    with pytest.raises(ValueError, match="y: shape"):
        B.experts_fwd(off, x, w, bf(10, 16))
    with pytest.raises(ValueError, match="row_token: shape"):
        B.experts_fwd(off, x, w, y, row_token=i32(9))
    with pytest.raises(ValueError, match="w2: shape"):
        B.experts_fwd(off, x, w, y, w2=bf(4, 16, 16), y2=y)
    with pytest.raises(ValueError, match="GPU tensors only"):
        B.experts_fwd(off, x, w, y)
    with pytest.raises(ValueError, match="dx: shape"):
        B.experts_bwd_x(off, y, w, bf(9, 16))
    with pytest.raises(ValueError, match="dw: torch.bfloat16"):
        B.experts_bwd_w(off, x, y, w)
    with pytest.raises(ValueError, match="pos: shape"):
        B.experts_plan(4, i32(3, 2), off, i32(6), i32(6))
    with pytest.raises(ValueError, match="weights: torch.bfloat16"):
        B.experts_combine_fwd(y, i32(5, 2), bf(5, 2), bf(5, 24))
    with pytest.raises(ValueError, match="dweights: shape"):
        B.experts_combine_bwd(bf(5, 24), y, i32(5, 2), None, y, torch.zeros(5, 1))


# sizes that 32 bits hold, but not what the kernels round them up to
@pytest.mark.parametrize("kw", [dict(rows=2147483647, x_rows=2147483647, i=8, o=8), dict(rows=2147483400, x_rows=2147483400, i=8, o=8),
                                dict(rows=2147482624, x_rows=2147482624, i=8, o=8),
                                dict(E=1, rows=1, i=2147483640, o=8), dict(E=1, rows=1, i=8, o=2147482624)])
def test_sizes_next_to_32_bits(kw):
    far = lambda *names: {n: 0x7F0000000000 + j * (1 << 40) for j, n in enumerate(names)}
    plain = {k: v for k, v in kw.items() if k != "x_rows"}
    for call, base, args in (("spr_experts_fwd", FWD, {**kw, **far("x", "w", "y", "w2", "y2", "offsets")}),
                             ("spr_experts_bwd_x", BWD_X, {**plain, **far("dy", "w", "dy2", "w2", "dx", "offsets")}),
                             ("spr_experts_bwd_w", BWD_W, {**kw, **far("x", "dy", "dw", "dy2", "dw2", "offsets")}),
                             ("spr_experts_bwd_w", BWD_W, {**kw, **far("x", "dy", "dw", "dy2", "dw2", "offsets", "row_token")})):
        assert _call(call, base, **args) == "SPR_ERR_INVALID_ARG", call
        assert "2^31 - 1025" in B.last_error()


def test_the_largest_widths_without_rows():
    most = 2147482616
    for i, o in ((most, 8), (8, most)):
        assert _call("spr_experts_fwd", FWD, E=1, rows=0, i=i, o=o) == "SPR_OK"
        assert _call("spr_experts_bwd_x", BWD_X, E=1, rows=0, i=i, o=o) == "SPR_OK"
        assert _call("spr_experts_bwd_w", BWD_W, E=1, rows=0, i=i, o=o, overwrite=0) == "SPR_OK"
