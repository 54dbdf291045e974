"""The products grouped by expert against the formulas in 64 bits.

An element is a sum of n products of bf16 values, exact in fp32 each, added in
fp32: at most 2^-23 of the sum of magnitudes per addition (twice half a step,
so that an addition that cuts off instead of rounding is counted too), and for
a bf16 result half a step of its own, 2^-8 of the value."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
HALF = 2.0 ** -8 * 1.001


def _say(what):
    print(f"\n[gpu experts] {what}", flush=True)


def _make(sizes, i, o, tokens=None, tail=0, seed=0):
    """Inputs of groups of the given sizes, `tail` further rows behind them;
    `tokens`: the rows of x that the sorted rows gather from."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    E, rows = len(sizes), sum(sizes) + tail
    off = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    tok = None
    if tokens is not None:
        tok = torch.randint(0, tokens, (rows,), generator=g, device="cuda").to(torch.int32)
        tok[sum(sizes):] = -1
    return dict(sizes=sizes, off=off, tok=tok, x=r(tokens if tokens is not None else rows, i), w=r(E, i, o),
                w2=r(E, i, o), dy=r(rows, o), dy2=r(rows, o))


def _groups(s):
    lo = 0
    for e, n in enumerate(s["sizes"]):
        yield e, slice(lo, lo + n)
        lo += n


def _rows_of_x(s, rows):
    x = s["x"].double()
    return x[rows] if s["tok"] is None else x[s["tok"][rows].long()]


def _within(got, ref, mag, n, half, what):
    off = (got.double() - ref).abs() - (half * ref.abs() + (n + 1) * U * mag)
    assert (off <= 0).all(), f"{what}: {off.max().item():.3e} over the bound"


def _check_all(s, i, o, two=True):
    import torch
    from paper_2606_01143_amd import binding as B
    rows, E = s["dy"].shape[0], len(s["sizes"])
    valid = sum(s["sizes"])
    new = lambda *sh, dt=torch.bfloat16: torch.full(sh, 3.0, dtype=dt, device="cuda")
    y, y2, dx, dx1 = new(rows, o), new(rows, o), new(rows, i), new(rows, i)
    B.experts_fwd(s["off"], s["x"], s["w"], y, w2=s["w2"] if two else None, y2=y2 if two else None,
                  row_token=s["tok"])
    B.experts_bwd_x(s["off"], s["dy"], s["w"], dx, dy2=s["dy2"] if two else None, w2=s["w2"] if two else None)
    B.experts_bwd_x(s["off"], s["dy2"], s["w2"], dx1)
    dw, dw2, add = (new(E, i, o, dt=torch.float32) for _ in range(3))
    B.experts_bwd_w(s["off"], s["x"], s["dy"], dw, dy2=s["dy2"] if two else None, dw2=dw2 if two else None,
                    row_token=s["tok"], overwrite=True)
    B.experts_bwd_w(s["off"], s["x"], s["dy"], add, row_token=s["tok"])
    torch.cuda.synchronize()
    for e, rs in _groups(s):
        x, w, w2 = _rows_of_x(s, rs), s["w"][e].double(), s["w2"][e].double()
        dy, dy2 = s["dy"][rs].double(), s["dy2"][rs].double()
        _within(y[rs], x @ w, x.abs() @ w.abs(), i, HALF, f"y of expert {e}")
        ref, mag, n = dy @ w.t(), dy.abs() @ w.abs().t(), o
        if two:
            _within(y2[rs], x @ w2, x.abs() @ w2.abs(), i, HALF, f"y2 of expert {e}")
            ref, mag, n = ref + dy2 @ w2.t(), mag + dy2.abs() @ w2.abs().t(), 2 * o
        _within(dx[rs], ref, mag, n, HALF, f"dx of expert {e}")
        _within(dx1[rs], dy2 @ w2.t(), dy2.abs() @ w2.abs().t(), o, HALF, f"one pair's dx of expert {e}")
        c = x.shape[0]
        _within(dw[e], x.t() @ dy, x.abs().t() @ dy.abs(), c, 0.0, f"dw of expert {e}")
        _within(add[e], x.t() @ dy + 3, x.abs().t() @ dy.abs() + 3, c + 1, 0.0, f"dw added, expert {e}")
        if two:
            _within(dw2[e], x.t() @ dy2, x.abs().t() @ dy2.abs(), c, 0.0, f"dw2 of expert {e}")
    # rows behind the last group, and what is not asked for, stay as they were
    for t in (y, dx, dx1) + ((y2,) if two else ()):
        assert (t[valid:] == 3).all()
    if not two:
        assert (y2 == 3).all() and (dw2 == 3).all()


SIZES = {"one_row": [1], "single_rows": [1, 0, 1, 1, 0, 0, 1, 1], "edges": [31, 32, 33, 0, 63, 64, 65],
         "tile_edges": [127, 128, 129, 0, 255, 256, 257], "one_group": [300], "skewed": [0, 700, 0, 3, 40, 0, 0, 9],
         "many": [int(v) for v in np.random.default_rng(0).integers(0, 9, 200)],
         "most": [0] * 700 + [5] + [0] * 322 + [2],
         "even": [96] * 16}


@pytest.mark.parametrize("i,o", [(64, 128), (8, 8), (40, 264), (520, 72), (136, 136), (256, 384)])
@pytest.mark.parametrize("name", ["one_row", "single_rows", "edges", "tile_edges", "skewed"])
def test_shapes(gpu, name, i, o):
    _say(f"{name} {i} x {o}")
    sizes = SIZES[name]
    _check_all(_make(sizes, i, o, tokens=50, tail=7, seed=i + o), i, o)


@pytest.mark.parametrize("name,i,o,tokens,two", [
    ("one_group", 128, 128, None, False), ("one_group", 1024, 48, 9, True), ("many", 72, 64, 33, True),
    ("most", 32, 40, None, True), ("even", 512, 256, 200, True), ("even", 256, 640, None, False),
    ("tile_edges", 768, 128, None, True)])
def test_groups(gpu, name, i, o, tokens, two):
    _say(f"{name} {i} x {o} tokens {tokens} two {two}")
    _check_all(_make(SIZES[name], i, o, tokens=tokens, tail=0 if tokens is None else 3, seed=1), i, o, two)


def test_no_rows(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    bf = dict(dtype=torch.bfloat16, device="cuda")
    off, w = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.randn(4, 16, 24, device="cuda").bfloat16()
    x, dy = torch.empty(0, 16, **bf), torch.empty(0, 24, **bf)
    B.experts_fwd(off, x, w, torch.empty(0, 24, **bf))
    B.experts_bwd_x(off, dy, w, torch.empty(0, 16, **bf))
    dw = torch.ones(4, 16, 24, device="cuda")
    B.experts_bwd_w(off, x, dy, dw)
    assert (dw == 1).all()
    B.experts_bwd_w(off, x, dy, dw, overwrite=True)
    assert (dw == 0).all()
    # rows, but none of them any expert's
    s = _make([0, 0, 0], 16, 24, tail=40)
    _check_all(s, 16, 24)


def test_no_rows_of_a_pair(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    bf = dict(dtype=torch.bfloat16, device="cuda")
    off, w = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.randn(4, 16, 24, device="cuda").bfloat16()
    x, dy, tokens = torch.empty(0, 16, **bf), torch.empty(0, 24, **bf), torch.empty(0, dtype=torch.int32, device="cuda")
    table = torch.ones(7, 16, **bf)
    for src, rt in ((x, None), (table, tokens)):
        B.experts_fwd(off, src, w, torch.empty(0, 24, **bf), w, torch.empty(0, 24, **bf), row_token=rt)
        dw, dw2 = torch.ones(4, 16, 24, device="cuda"), torch.ones(4, 16, 24, device="cuda")
        B.experts_bwd_w(off, src, dy, dw, dy, dw2, row_token=rt)
        assert (dw == 1).all() and (dw2 == 1).all()
        B.experts_bwd_w(off, src, dy, dw, dy, dw2, row_token=rt, overwrite=True)
        assert (dw == 0).all() and (dw2 == 0).all()
    B.experts_bwd_x(off, dy, w, x, dy, w)


def test_a_bad_row_stays_in_its_group(gpu):
    """NaN and infinity in one expert's last row, its weights or the rows
    behind the last group reach nothing else; ragged contraction ends too."""
    import torch
    from paper_2606_01143_amd import binding as B
    i, o = 40, 72
    s = _make([33, 20, 0, 45], i, o, tail=5, seed=3)
    bad = {n: t.clone() for n, t in s.items() if n in ("x", "dy", "w")}
    last = 33 + 20 - 1
    bad["x"][last, 39], bad["dy"][last, 71] = float("inf"), float("nan")
    bad["x"][-5:], bad["dy"][-5:] = float("nan"), float("inf")
    bad["w"][3, 39, 0] = float("nan")
    out = []
    for t in (s, {**s, **bad}):
        y, dx = torch.zeros(103, o, device="cuda").bfloat16(), torch.zeros(103, i, device="cuda").bfloat16()
        dw = torch.zeros(4, i, o, device="cuda")
        B.experts_fwd(t["off"], t["x"], t["w"], y)
        B.experts_bwd_x(t["off"], t["dy"], t["w"], dx)
        B.experts_bwd_w(t["off"], t["x"], t["dy"], dw)
        out.append((y, dx, dw))
    (y0, dx0, dw0), (y, dx, dw) = out
    assert not torch.isfinite(y[last]).any() and dx[last].isnan().all()
    assert y[53:98, 0].isnan().all() and dx[53:98, 39].isnan().all()
    assert torch.equal(y[53:98, 1:], y0[53:98, 1:]) and torch.equal(dx[53:98, :39], dx0[53:98, :39])
    assert torch.equal(y[:last], y0[:last]) and torch.equal(dx[:last], dx0[:last])
    assert torch.equal(dw[[0, 2, 3]], dw0[[0, 2, 3]])
    assert torch.equal(dw[1, :39, :71], dw0[1, :39, :71]) and not torch.isfinite(dw[1, 39]).any()
    assert dw[1, :, 71].isnan().all()


def test_wrong_offsets_and_tokens_stay_inside(gpu):
    """Offsets out of order or range and tokens out of range are clamped: the
    calls end, groups that are right are right, and nothing is written
    behind the outputs."""
    import torch
    from paper_2606_01143_amd import binding as B
    i, o, rows = 64, 128, 90
    s = _make([30, 30, 30], i, o, tokens=20, seed=4)
    off = torch.tensor([0, 30, -5, 1 << 30], dtype=torch.int32, device="cuda")
    tok = s["tok"].clone()
    tok[:3] = torch.tensor([-7, 20, 2147483647], dtype=torch.int32)
    buf = torch.full((rows + 64, o), 3.0, device="cuda").bfloat16()
    B.experts_fwd(off, s["x"], s["w"], buf[:rows], row_token=tok)
    dw = torch.zeros(4, i, o, device="cuda")
    dw[3] = 5
    B.experts_bwd_w(off, s["x"], s["dy"], dw[:3], row_token=tok)
    torch.cuda.synchronize()
    assert (buf[rows:] == 3).all() and (dw[3] == 5).all()
    x = s["x"].double()[tok[3:30].long()]
    ref = x @ s["w"][0].double()
    # rows 3 .. 29 are the first group's alone unless a later group overlaps it: the third group is
    # offsets -5 .. 2^30, that is all the rows, so each row is one of the two experts' products
    other = x @ s["w"][2].double()
    mag = x.abs() @ s["w"].double().abs().amax(0)
    off1, off2 = (((buf[3:30].double() - r).abs() - (HALF * r.abs() + (i + 1) * U * mag)).amax(1) for r in (ref, other))
    assert torch.minimum(off1, off2).max() <= 0


def test_far_rows_and_weights(gpu):
    """Byte offsets past 32 bits, in the rows and in the weights."""
    import torch
    from paper_2606_01143_amd import binding as B
    _say("far rows")
    i, o, n = 2048, 16, 1100000
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(n, i, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(2, i, o, generator=g, device="cuda", dtype=torch.bfloat16)
    off = torch.tensor([0, 70, n], dtype=torch.int32, device="cuda")
    y = torch.empty(n, o, dtype=torch.bfloat16, device="cuda")
    B.experts_fwd(off, x, w, y)
    dx = torch.empty_like(x)
    B.experts_bwd_x(off, y, w, dx)
    tail = slice(n - 300, n)
    xt = x[tail].double()
    _within(y[tail], xt @ w[1].double(), xt.abs() @ w[1].double().abs(), i, HALF, "far y")
    yt = y[tail].double()
    _within(dx[tail], yt @ w[1].double().t(), yt.abs() @ w[1].double().abs().t(), o, HALF, "far dx")
    del x, y, dx, w
    _say("far weights")
    E, i, o = 300, 4096, 2048
    w = torch.zeros(E, i, o, dtype=torch.bfloat16, device="cuda")
    w[-1] = torch.randn(i, o, generator=g, device="cuda")
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[-1] = 40
    x = torch.randn(40, i, generator=g, device="cuda").bfloat16()
    y, dx = torch.empty(40, o, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    B.experts_fwd(off, x, w, y)
    B.experts_bwd_x(off, y, w, dx)
    wd = w[-1].double()
    _within(y, x.double() @ wd, x.double().abs() @ wd.abs(), i, HALF, "far weights' y")
    _within(dx, y.double() @ wd.t(), y.double().abs() @ wd.abs().t(), o, HALF, "far weights' dx")
    dw = torch.empty(E, i, o, device="cuda")
    B.experts_bwd_w(off, x, y, dw, overwrite=True)
    _within(dw[-1], x.double().t() @ y.double(), x.double().abs().t() @ y.double().abs(), 40, 0.0, "far dw")
    assert not dw[:-1].any()


def test_gradients_are_the_products_derivatives(gpu):
    """Differences of the loss <dy, y> in 64 bits, in single weights and rows,
    from the kernels' own operands."""
    import torch
    from paper_2606_01143_amd import binding as B
    s = _make([5, 0, 9], 16, 24, tokens=6, seed=6)
    rows = 14
    dx, dw = torch.empty(rows, 16, device="cuda").bfloat16(), torch.empty(3, 16, 24, device="cuda")
    B.experts_bwd_x(s["off"], s["dy"], s["w"], dx)
    B.experts_bwd_w(s["off"], s["x"], s["dy"], dw, row_token=s["tok"], overwrite=True)

    def loss(x, w):
        return sum((s["dy"][rs].double() * (x[rs] @ w[e])).sum() for e, rs in _groups(s))
    x, w = s["x"].double()[s["tok"].long()], s["w"].double()
    for at in [(0, 3), (4, 15), (13, 0)]:
        d = torch.zeros_like(x)
        d[at] = 0.5
        want = (loss(x + d, w) - loss(x - d, w)).item()
        mag = (s["dy"][at[0]].double().abs().sum() * s["w"].double().abs().max()).item()
        assert abs(dx[at].item() - want) <= HALF * abs(want) + 26 * U * mag
    for at in [(0, 0, 0), (0, 15, 23), (2, 7, 9), (1, 2, 2)]:
        d = torch.zeros_like(w)
        d[at] = 0.5
        want = (loss(x, w + d) - loss(x, w - d)).item()
        assert abs(dw[at].item() - want) <= 16 * U * rows * 16


def test_repeats_streams_and_graphs(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    _say("graph")
    side = torch.cuda.Stream()
    caught = []
    for sizes, i, o in (([40, 0, 200, 7], 136, 264), ([1, 0, 2], 64, 64)):
        s = _make(sizes, i, o, tokens=30, seed=7)
        rows = sum(sizes)
        bf = dict(dtype=torch.bfloat16, device="cuda")

        def call(y, dx, dw, stream=None, s=s):
            B.experts_fwd(s["off"], s["x"], s["w"], y, row_token=s["tok"], stream=stream)
            B.experts_bwd_x(s["off"], s["dy"], s["w"], dx, dy2=s["dy2"], w2=s["w2"], stream=stream)
            B.experts_bwd_w(s["off"], s["x"], s["dy"], dw, row_token=s["tok"], overwrite=True, stream=stream)
        outs = [(torch.empty(rows, o, **bf), torch.empty(rows, i, **bf), torch.empty(len(sizes), i, o, device="cuda"))
                for _ in range(3)]
        call(*outs[0])
        side.wait_stream(torch.cuda.current_stream())
        call(*outs[1], stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[1]))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(*outs[2])
        caught.append((graph, outs, s, call))
    for _ in range(4):
        for graph, outs, s, call in caught:
            for t in outs[2]:
                t.fill_(9)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[0], outs[2]))
            call(*outs[1])


def _raised(off, rows):
    return np.maximum.accumulate(np.clip(off, 0, rows))


@pytest.mark.parametrize("name,i,o", [
    ("back", 64, 128), ("back", 256, 384), ("many", 72, 64), ("most", 40, 136), ("large", 264, 264), ("first", 64, 64),
    ("large", 1024, 2056)])
def test_offsets_out_of_order_are_raised(gpu, name, i, o):
    """Bitwise what the clamped offsets' running maximum gives: no row belongs to
    two experts, and none that it gives to one is left out."""
    import torch
    from paper_2606_01143_amd import binding as B
    _say(f"raised {name} {i} x {o}")
    rng = np.random.default_rng(i)
    noisy = lambda E, rows: np.sort(rng.integers(0, rows, E + 1)) + rng.integers(-rows // 3, 1, E + 1)
    rows, off = {"back": (90, [0, 30, -5, 1 << 30]), "many": (500, noisy(200, 500)),
                 "most": (700, [*noisy(1022, 700), -2147483648, 2147483647]), "first": (70, [50, 0, 20, 60, 60, 10]),
                 "large": (2600, [0, 900, 400, 1500, 1400, -1, 2300, 2147483647, 0])}[name]
    off = np.array(off)
    want = _raised(off, rows)
    s = _make([rows], i, o, tokens=60, seed=i)
    E = len(off) - 1
    g = torch.Generator(device="cuda").manual_seed(o)
    w, w2 = (torch.randn(E, i, o, generator=g, device="cuda").bfloat16() for _ in range(2))
    new = lambda *sh, dt=torch.bfloat16: torch.full(sh, 3.0, dtype=dt, device="cuda")
    outs = []
    for f in (want, off, off):
        t = torch.from_numpy(f.astype(np.int32)).cuda()
        r = [new(rows, o), new(rows, o), new(rows, i), new(rows, i), *(new(E, i, o, dt=torch.float32) for _ in range(4))]
        B.experts_fwd(t, s["x"], w, r[0], w2=w2, y2=r[1], row_token=s["tok"])
        B.experts_bwd_x(t, s["dy"], w, r[2], dy2=s["dy2"], w2=w2)
        B.experts_bwd_x(t, s["dy"], w, r[3])
        B.experts_bwd_w(t, s["x"], s["dy"], r[4], dy2=s["dy2"], dw2=r[5], row_token=s["tok"], overwrite=True)
        xs = s["x"][s["tok"].long()]
        B.experts_bwd_w(t, xs, s["dy"], r[6])
        B.experts_bwd_w(t, xs, s["dy"], r[7], overwrite=True)
        torch.cuda.synchronize()
        outs.append(r)
    for r in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], r))
    # and the raised offsets are the groups of the formula
    y, dw = outs[1][0], outs[1][4]
    for e in range(E):
        a, b = want[e], want[e + 1]
        x, dy = s["x"].double()[s["tok"][a:b].long()], s["dy"][a:b].double()
        _within(y[a:b], x @ w[e].double(), x.abs() @ w[e].double().abs(), i, HALF, f"y of expert {e}")
        _within(dw[e], x.t() @ dy, x.abs().t() @ dy.abs(), b - a, 0.0, f"dw of expert {e}")
    assert (y[:want[0]] == 3).all() and (y[want[-1]:] == 3).all()
