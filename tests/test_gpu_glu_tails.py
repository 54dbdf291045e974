"""The gated feed-forward's activations and slopes against 64 bits, relative to
their own size, tails included.

Both activations are g s with s the sigmoid of z (z = g, or 2 sqrt(2 / pi) (g +
0.044715 g^3)); U = 2^-23 is a step of fp32.  z's own roundings are at most 2.5 U
of it, exp's of an argument z 0.75 U |z| and 1.5 U more, the sum, its reciprocal
and the product 2 U: s and g s are right to R = 4 U (1 + |z|), relative.  Behind z =
-87 s is below 2^-126 and may be 0: with |g| < 128 there (s is 0 in both forms where
g < -104) an absolute 2^-119 is allowed for.
The slope is s + g (1 - s) s z'.  1 - s carries s's absolute error and a rounding (R s
+ U where z < 0, 3 U where z > 0; from z = 17 on fp32 has s = 1, and next to it the
term is off by no more than its own size), relative to |g s z'|.  |z'| < 512 where s is not 0: 2^-110."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
HALF = 2.0 ** -8


def _all(kind):
    """Every eighth finite bf16 of both signs (every exponent, 16 fractions of each),
    and in 64 bits the activation, its slope and their bounds."""
    bits = torch.arange(0, 65536, 8, device="cuda").to(torch.int32) << 16
    g = bits.view(torch.float32).bfloat16()
    g = torch.where(torch.isfinite(g), g, torch.ones_like(g))
    x = g.double()
    k = 2 * math.sqrt(2 / math.pi)
    if kind == "silu":
        z, dz = x, torch.ones_like(x)
    else:
        z, dz = k * (x + 0.044715 * x ** 3), k * (1 + 3 * 0.044715 * x * x)
    s, c = torch.sigmoid(z), torch.sigmoid(-z)
    rel = 4 * U * (1 + z.abs().clamp(max=1e4))
    value, term = torch.where(s == 0, 0.0, x * s), torch.where((s == 0) | (c == 0), 0.0, x * s * c * dz)
    value_err = rel * value.abs() + 2.0 ** -119
    c_err = torch.where(z < 0, rel * s + U, 3 * U)
    of_c = torch.where(z < 16, c_err * torch.where(s == 0, 0.0, x * s * dz).abs(), term.abs())
    return g, (value, value_err), (s + term, rel * (s + term.abs()) + of_c + 2.0 ** -110)


def _near(got, ref, what):
    ref, err = ref
    err = err + HALF * (ref.abs() + err)  # and one rounding to bf16
    off = (got.double() - ref).abs() - err
    i = off.argmax()
    assert torch.isfinite(got).all() and (off <= 0).all(), f"{what}: {got[i]} instead of {ref[i]}, allowed {err[i]}"


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_backward(gpu, kind):
    """dm and u are ones: dg is the slope, du and m the activation."""
    from paper_2606_01143_amd import binding as B
    print(f"\n[gpu glu] tails, backward {kind}", flush=True)
    g, value, slope = _all(kind)
    # rows of 8 columns, and one row of all of them
    for shape in ((-1, 8), (1, -1)):
        gs = g.view(shape).contiguous()
        rows, mid = gs.shape
        one = torch.ones(rows, mid, dtype=torch.bfloat16, device="cuda")
        dy, wd = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(mid, 8, dtype=torch.bfloat16, device="cuda")
        dy[:, 0], wd[:, 0] = 1, 1
        dg, du, m = (torch.empty_like(one) for _ in range(3))
        B.glu_bwd(dy, wd, gs, one, dg, du, m=m, act=kind)
        _near(dg.view(-1), slope, "dg")
        _near(du.view(-1), value, "du")
        _near(m.view(-1), value, "m")


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("rows", [1, 300])
def test_forward(gpu, rows, kind):
    """x's first column is one and the others zeros: g is w_gate's first row, u ones."""
    from paper_2606_01143_amd import binding as B
    print(f"\n[gpu glu] tails, forward {rows} {kind}", flush=True)
    g, value, _ = _all(kind)
    x = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    wg, wu = (torch.zeros(8, g.numel(), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x[:, 0], wg[0], wu[0] = 1, g, 1
    m = torch.empty(rows, g.numel(), dtype=torch.bfloat16, device="cuda")
    B.glu_fwd(x, wg, wu, m, act=kind)
    for row in (0, rows - 1):
        _near(m[row], value, f"m, row {row}")
