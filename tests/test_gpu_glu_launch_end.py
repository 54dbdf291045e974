"""The gated feed-forward at a size whose tiles of 64 rows are more than a launch
holds: 60 experts of 8 x 2^24, 384 rows, some experts without any (45 GB), against
64 bits in sampled columns, with test_gpu_glu's bounds."""
import pytest
import torch

from test_gpu_glu import HALF, SLOPE, U, act
from test_glu_launch_sizes import FWD, MOST, threads

pytestmark = pytest.mark.gpu


def test_tiles_of_64_rows_do_not_fit(gpu):
    from paper_2606_01143_amd import binding as B
    E, rows, K, N = 60, 384, 8, 1 << 24
    assert threads(FWD[0], E, rows, N) > MOST
    print(f"\n[gpu glu] {E} experts, {rows} rows, {K} x {N}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(0)
    sizes = [0, 1, 64, 3, 0, 65] + [1] * 40 + [15] * 13 + [16]
    assert len(sizes) == E and sum(sizes) == rows
    off = torch.tensor([0] + sizes, device="cuda").cumsum(0).to(torch.int32)
    x = torch.randn(rows, K, generator=g, device="cuda").bfloat16()
    wg, wu = (torch.empty(E, K, N, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    m = torch.full((rows, N), 3.0, dtype=torch.bfloat16, device="cuda")
    B.glu_fwd(x, wg, wu, m, offsets=off)
    torch.cuda.synchronize()
    at = torch.cat([torch.arange(64), torch.randint(0, N, (4000,), generator=torch.Generator().manual_seed(1)),
                    torch.arange(N - 64, N)]).cuda()
    for e, (lo, hi) in enumerate(zip(off.tolist(), off.tolist()[1:])):
        if lo == hi:
            continue
        xs, a, b = x[lo:hi].double(), wg[e][:, at].double(), wu[e][:, at].double()
        rg, ru, eg, eu = xs @ a, xs @ b, (K + 1) * U * (xs.abs() @ a.abs()), (K + 1) * U * (xs.abs() @ b.abs())
        value = act("silu", rg)[0]
        err = (SLOPE * eg + 32 * U * rg.abs()) * (ru.abs() + eu) + value.abs() * eu
        off_by = (m[lo:hi][:, at].double() - value * ru).abs() - HALF * (value * ru).abs() - err - 1e-37
        assert (off_by <= 0).all(), (e, off_by.max().item())
    del wg, wu, m
    torch.cuda.empty_cache()
