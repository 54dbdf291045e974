"""Infinite gains and gates in the norms' backward: the gradients that the formulas
make infinite are infinite, whatever the number of rows (a workgroup holds
several rows at once, and the last one's places may be empty)."""
import pytest
import torch

from test_gpu_block import C, U, _types

pytestmark = pytest.mark.gpu

INF = float("inf")


def _positive(rows, width, dt, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (0.5 + torch.rand(rows, width, generator=g, device="cuda")).to(dt)


def _bwd(rows, width, dt, gain_pre, gate):
    from paper_2606_01143_amd import binding as B
    h, f, dn = (_positive(rows, width, dt, s) for s in (1, 2, 3))
    rh, rf = (t.float().square().mean(1).rsqrt() for t in (h, f))
    dx, df = torch.empty_like(h), torch.empty_like(h)
    post, pre = (torch.full((width,), 7.0, device="cuda") for _ in range(2))
    dgate = torch.full((width,), 7.0, device="cuda") if gate.dim() == 1 else torch.empty_like(gate)
    ws = torch.empty(B.block_norm_bwd_workspace_size(rows, width), dtype=torch.uint8, device="cuda")
    B.block_norm_bwd(h, f, None, dn, dx, df, rstd_f=rf, rstd_h=rh, gate=gate, gain_pre=gain_pre, dgain_post=post,
                     dgate=dgate, dgain_pre=pre, overwrite=True, ws=ws)
    return h, f, dn, rh.double()[:, None], rf.double()[:, None], dx, post, dgate, pre


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 3, 8, 9])
@pytest.mark.parametrize("width", [64, 1000, 2048])
def test_an_infinite_gain(gpu, width, rows, dtype):
    """Column 5's gain is infinite.  With h, f and dn positive the rows' k = r_h^3
    mean(gain dn h) is infinite, d = r_h gain dn - k h is -inf (NaN in column 5,
    inf - inf), and so are the sums of d f r_f."""
    print(f"\n[gpu block] infinite gain {rows} x {width} {dtype}", flush=True)
    dt = _types()[dtype]
    gain = torch.ones(width, dtype=dt, device="cuda")
    gain[5] = INF
    h, f, dn, rh, rf, dx, post, dgate, pre = _bwd(rows, width, dt, gain, torch.ones(width, dtype=dt, device="cuda"))
    rest = torch.arange(width, device="cuda") != 5
    for t in (dx, post[None], dgate[None]):
        assert torch.isneginf(t[:, rest]).all()
        assert torch.isnan(t[:, 5]).all()
    ref = (dn.double() * h.double() * rh).sum(0)  # no gain in it, all terms positive
    assert ((pre.double() - ref).abs() <= (C + rows) * U * ref).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_gate_of_one_row(gpu, dtype):
    """Row 3's own gate is infinite in column 7, and only that column's sum of
    gate d f r_f is: 4097 rows of 64 are one more than the rows that all
    workgroups hold at once, so that row 3's place is empty in the last turn."""
    print(f"\n[gpu block] infinite gate {dtype}", flush=True)
    dt, rows, width = _types()[dtype], 4097, 64
    gate = torch.ones(rows, width, dtype=dt, device="cuda")
    gate[3, 7] = INF
    h, f, dn, rh, rf, dx, post, dgate, pre = _bwd(rows, width, dt, None, gate)
    hd, td = h.double(), dn.double()
    d = rh * td - hd * rh ** 3 * (td * hd).mean(1, keepdim=True)
    terms = d * f.double() * rf
    ref, mag = terms.sum(0), (rh * td * f.double() * rf).sum(0) * 2
    assert torch.isinf(post[7]) and torch.signbit(post[7]) == torch.signbit(d[3, 7])
    rest = torch.arange(width, device="cuda") != 7
    assert ((post.double() - ref).abs() <= (C + rows) * U * mag)[rest].all()
    assert torch.isfinite(dx).all() and torch.isfinite(dgate).all()
