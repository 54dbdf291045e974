"""Refusals of the per-head norm with rotation and of the embedding (CPU): bad
sizes, types, strides, alignment, overlaps and workspaces are turned away
before anything is launched.  The addresses are never dereferenced."""
import pytest
import torch

from paper_2606_01143_amd import binding as B

A = 0x7F0000000000


def _at(i, off=0):
    return A + i * (1 << 32) + off


def _heads_bwd(**kw):
    a = dict(dtype=1, T=10, hq=4, hkv=2, d=64, eps=1e-6, pos0=0, pos=None, theta=1e4, q=_at(1), qs=512, k=_at(1, 512),
             ks=512, gq=_at(2), gk=_at(3), dyq=_at(4), dyk=_at(5), dq=_at(6), dqs=512, dk=_at(6, 512), dks=512,
             dgq=_at(7), dgk=_at(8), ow=1, ws=_at(9), wsb=1 << 30)
    a.update(kw)
    return B.STATUS[B.lib().spr_head_norm_rope_bwd(*a.values(), None)]


def _heads_fwd(**kw):
    a = dict(dtype=1, T=10, hq=4, hkv=2, d=64, eps=1e-6, pos0=0, pos=None, theta=1e4, q=_at(1), qs=512, k=_at(1, 512),
             ks=512, gq=_at(2), gk=_at(3), yq=_at(4), yk=_at(5))
    a.update(kw)
    return B.STATUS[B.lib().spr_head_norm_rope_fwd(*a.values(), None)]


SIZES = [(dict(dtype=2), "UNSUPPORTED"), (dict(T=-1), "INVALID_ARG"), (dict(hq=0), "INVALID_ARG"),
         (dict(hkv=0), "INVALID_ARG"), (dict(d=63), "UNSUPPORTED"), (dict(d=258), "UNSUPPORTED"),
         (dict(d=0), "UNSUPPORTED"), (dict(eps=-1.0), "INVALID_ARG"), (dict(eps=float("nan")), "INVALID_ARG"),
         (dict(eps=float("inf")), "INVALID_ARG"), (dict(pos0=-1), "INVALID_ARG"), (dict(theta=1.0), "INVALID_ARG"),
         (dict(theta=float("inf")), "INVALID_ARG"), (dict(qs=255), "INVALID_ARG"), (dict(ks=127), "INVALID_ARG"),
         (dict(qs=1 << 40), "INVALID_ARG"), (dict(T=1 << 30), "INVALID_ARG"),
         (dict(T=1, hq=1 << 25, qs=1 << 31), "INVALID_ARG"), (dict(q=None), "INVALID_ARG"),
         (dict(gk=None), "INVALID_ARG"), (dict(q=_at(1, 1)), "MISALIGNED"), (dict(gq=_at(2, 1)), "MISALIGNED"),
         (dict(pos=_at(20, 2)), "MISALIGNED")]


@pytest.mark.parametrize("kw,status", SIZES)
def test_heads_sizes(kw, status):
    assert _heads_fwd(**kw) == "SPR_ERR_" + status
    assert B.last_error()
    assert _heads_bwd(**kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", [
    (dict(yq=_at(4, 2)), "MISALIGNED"), (dict(yk=None), "INVALID_ARG"), (dict(yq=_at(1)), "ALIASING"),
    (dict(yk=_at(4, 64)), "ALIASING"), (dict(yq=_at(2)), "ALIASING")])
def test_heads_forward_outputs(kw, status):
    assert _heads_fwd(**kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", [
    (dict(dyq=_at(4, 2)), "MISALIGNED"), (dict(dgq=_at(7, 2)), "MISALIGNED"), (dict(dgk=None), "INVALID_ARG"),
    (dict(dq=_at(1)), "ALIASING"),                  # the gradient on q itself
    (dict(dk=_at(6, 510)), "ALIASING"),             # one element of dq's last head
    (dict(dk=_at(6, 512), dks=520), "ALIASING"),    # two strides in one buffer
    (dict(dk=_at(6, 770)), "ALIASING"),             # its end in the next token's dq
    (dict(dq=_at(4)), "ALIASING"), (dict(dgq=_at(6)), "ALIASING"), (dict(dgq=_at(8)), "ALIASING"),
    (dict(ws=_at(6)), "ALIASING"), (dict(ws=_at(1)), "ALIASING"), (dict(ws=None), "WORKSPACE"),
    (dict(wsb=16), "WORKSPACE"), (dict(ws=_at(9, 4)), "MISALIGNED"), (dict(dqs=255), "INVALID_ARG")])
def test_heads_backward_outputs(kw, status):
    assert _heads_bwd(**kw) == "SPR_ERR_" + status


def test_heads_workspace_size():
    assert B.head_norm_rope_bwd_workspace_size(1, 1, 1, 2) > 0
    with pytest.raises(B.SprError):
        B.head_norm_rope_bwd_workspace_size(10, 4, 2, 65)
    out = B.lib().spr_head_norm_rope_bwd_workspace_size(10, 4, 2, 64, None)
    assert B.STATUS[out] == "SPR_ERR_INVALID_ARG"


def _embed(fwd, **kw):
    a = dict(dtype=1, T=10, V=100, w=64, scale=1.0, ids=_at(1), x=_at(2), y=_at(3))
    ws = dict(ws=_at(4), wsb=1 << 30)
    ws.update({k: kw.pop(k) for k in list(kw) if k in ws})
    a.update(kw)
    if fwd:
        return B.STATUS[B.lib().spr_embed_fwd(*a.values(), None)]
    return B.STATUS[B.lib().spr_embed_bwd(*a.values(), *ws.values(), None)]


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), "UNSUPPORTED"), (dict(T=-1), "INVALID_ARG"), (dict(V=0), "INVALID_ARG"),
    (dict(w=12), "UNSUPPORTED"), (dict(w=0), "UNSUPPORTED"), (dict(scale=float("nan")), "INVALID_ARG"),
    (dict(ids=None), "INVALID_ARG"), (dict(ids=_at(1, 2)), "MISALIGNED"), (dict(x=_at(2, 8)), "MISALIGNED"),
    (dict(y=None), "INVALID_ARG"), (dict(y=_at(2)), "ALIASING"), (dict(y=_at(1)), "ALIASING"),
    (dict(T=2147483647, w=1 << 20), "INVALID_ARG")])
def test_embed_refusals(kw, status):
    assert _embed(True, **kw) == "SPR_ERR_" + status
    assert _embed(False, **kw) == "SPR_ERR_" + status


@pytest.mark.parametrize("kw,status", [(dict(ws=None), "WORKSPACE"), (dict(wsb=64), "WORKSPACE"),
                                       (dict(ws=_at(4, 8)), "MISALIGNED"), (dict(ws=_at(3)), "ALIASING"),
                                       (dict(ws=_at(1)), "ALIASING")])
def test_embed_workspace(kw, status):
    assert _embed(False, T=300, **kw) == "SPR_ERR_" + status  # up to 256 tokens need no workspace
    assert B.embed_bwd_workspace_size(256, 100, 64) == 0 < B.embed_bwd_workspace_size(257, 100, 64)


def _cpu(*shape, dt=torch.bfloat16):
    return torch.zeros(*shape, dtype=dt)


def test_binding_types_and_shapes():
    q, k, g = _cpu(3, 4, 64), _cpu(3, 2, 64), _cpu(64)
    fwd = lambda **kw: B.head_norm_rope_fwd(**{**dict(q=q, k=k, gain_q=g, gain_k=g, yq=_cpu(3, 4, 64),
                                                      yk=_cpu(3, 2, 64), pos0=0, theta=1e4), **kw})
    with pytest.raises(ValueError, match="q: torch.float16"):
        fwd(q=q.half())
    with pytest.raises(ValueError, match="k: torch.float32"):
        fwd(k=k.float())
    with pytest.raises(ValueError, match="gain_q: shape"):
        fwd(gain_q=_cpu(63))
    with pytest.raises(ValueError, match="yk: shape"):
        fwd(yk=_cpu(2, 2, 64))
    with pytest.raises(ValueError, match="positions: torch.int64"):
        fwd(positions=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="positions: shape"):
        fwd(positions=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU tensors only"):
        fwd()
    ids, t = torch.zeros(3, dtype=torch.int32), _cpu(9, 16)
    with pytest.raises(ValueError, match="ids: torch.int64"):
        B.embed_fwd(ids.long(), t, _cpu(3, 16))
    with pytest.raises(ValueError, match="table: torch.float16"):
        B.embed_fwd(ids, t.half(), _cpu(3, 16))
    with pytest.raises(ValueError, match="y: shape"):
        B.embed_fwd(ids, t, _cpu(3, 8))
    with pytest.raises(ValueError, match="dtable: torch.bfloat16"):
        B.embed_bwd(ids, _cpu(3, 16), t)
    with pytest.raises(ValueError, match="dy: shape"):
        B.embed_bwd(ids, _cpu(4, 16), t.float())


class _Cuda:
    """A tensor that claims to lie on a GPU."""
    is_cuda = True

    def __init__(self, shape, strides, dt=torch.bfloat16, index=0):
        self.shape, self._s, self.dtype, self.index = shape, strides, dt, index

    def stride(self):
        return self._s

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return _at(1)


def _rows(shape, strides):
    return B._rows_arg("q", _Cuda(shape, strides), torch.bfloat16, shape, 0)


def test_binding_strides_and_device(monkeypatch):
    assert _rows((5, 4, 64), (512, 64, 1)) == (_at(1), 512)
    assert _rows((1, 4, 64), (3, 64, 1)) == (_at(1), 256)
    assert _rows((5, 1, 64), (64, 7, 1)) == (_at(1), 64)
    with pytest.raises(ValueError, match="not contiguous"):
        _rows((5, 4, 64), (512, 128, 1))
    with pytest.raises(ValueError, match="not contiguous"):
        _rows((5, 4, 64), (512, 1, 4))
    with pytest.raises(ValueError, match="tokens overlap"):
        _rows((5, 4, 64), (0, 64, 1))
    bf = torch.bfloat16
    assert B._arg("q", _Cuda((2,), (1,)), bf, (2,), 0) == _at(1)
    with pytest.raises(ValueError, match="q is on cuda:1, not on the call's device cuda:0"):
        B._arg("q", _Cuda((2,), (1,), index=1), bf, (2,), 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="the tensors are on cuda:1, not on the current device cuda:0"):
        B._on(1, 5)
    assert B._on(0, 5) == 5


def test_embed_sizes_that_a_launch_holds():
    """2^39 values are still taken (their NULL pointer is not), more are not."""
    for fwd in (True, False):
        assert _embed(fwd, T=1 << 27, w=4096, ids=None) == "SPR_ERR_INVALID_ARG" and "ids" in B.last_error()
        assert _embed(fwd, T=(1 << 27) + 1, w=4096, ids=None) == "SPR_ERR_INVALID_ARG" and "2^39" in B.last_error()


def test_heads_strides():
    """Up to 2^31 - 1 elements, which a token's own heads may have; the refusal
    names the limit that was passed."""
    far = dict(q=A, k=A + (1 << 44), T=2, gq=None)  # the NULL gain is found behind the strides
    most = 2147483647
    assert _heads_fwd(**far, qs=most, ks=1 << 30) == "SPR_ERR_INVALID_ARG" and "gain_q" in B.last_error()
    assert _heads_bwd(**far, qs=most, ks=1 << 30, dqs=1 << 29, dks=most) == "SPR_ERR_INVALID_ARG"
    assert "gain_q" in B.last_error()
    for kw in (dict(qs=most + 1), dict(ks=1 << 40)):
        assert _heads_fwd(**{**far, **kw}) == "SPR_ERR_INVALID_ARG" and "exceeds 2^31 - 1" in B.last_error()
    assert _heads_fwd(qs=255) == "SPR_ERR_INVALID_ARG" and "at least" in B.last_error()
