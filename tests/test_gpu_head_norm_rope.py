"""Per-head norm and rotation against the formulas in 64 bits.

Tolerances count roundings (half a step each: 2^-24 in fp32, 2^-8 for the one
rounding of a bf16 output).  A rotated value p cos - q sin has at most 32 fp32
roundings on its way (the sum of squares' chain of up to 20, halved by the root,
the root, two products, the angle's half turns and its sine and cosine, the
rotation), each relative to |p| + |q|; the angle itself is formed in 64 bits and
is off by 2^-53 of its 8 steps at the position.  dx doubles that; a gain
gradient's sums are at most 256 terms deep at these sizes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
THETA = 500000.0


def _say(what):
    print(f"\n[gpu head norm rope] {what}", flush=True)


def _inputs(T, hq, hkv, d, dt, seed, extra=0, lead=0, positions=None):
    """q and k as views of one fused buffer of (hq + 2 hkv) heads and `extra`
    further elements a token, `lead` elements into it."""
    import torch
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).to(dt)
    width = (hq + 2 * hkv) * d + extra
    buf = r(T * width + lead).cuda()
    x = buf[lead:].view(T, width)
    cut = lambda b, a, n: b[:, a * d:(a + n) * d].unflatten(1, (n, d))
    return dict(x=x, q=cut(x, 0, hq), k=cut(x, hq, hkv), gq=(1 + 0.3 * r(d)).to(dt).cuda(),
                gk=(1 + 0.3 * r(d)).to(dt).cuda(), dyq=r(T, hq, d).cuda(), dyk=r(T, hkv, d).cuda(),
                pos=None if positions is None else torch.tensor(positions, dtype=torch.int32).cuda(), cut=cut)


def _ref(x, g, dy, pos, eps, theta=THETA):
    """y, dx, dg and the magnitudes their errors are relative to, in 64 bits."""
    x, g, dy = (t.double().cpu().numpy() for t in (x, g, dy))
    d = x.shape[-1]
    h = d // 2
    ang = pos[:, None, None] * theta ** (-2.0 * np.arange(h) / d)
    c, s = np.cos(ang), np.sin(ang)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    z = x * r * g
    a, b = z[..., :h], z[..., h:]
    y = np.concatenate([a * c - b * s, b * c + a * s], -1)
    mag = np.tile(np.abs(a) + np.abs(b), 2)
    a, b = dy[..., :h], dy[..., h:]
    dz = np.concatenate([a * c + b * s, b * c - a * s], -1)
    dmag = np.tile(np.abs(a) + np.abs(b), 2)
    gz = g * dz
    dx = r * gz - x * r ** 3 * (gz * x).mean(-1, keepdims=True)
    dxmag = r * np.abs(g) * dmag + np.abs(x) * r ** 3 * (np.abs(g) * dmag * np.abs(x)).mean(-1, keepdims=True)
    dg = (dz * x * r).sum((0, 1))
    dgmag = (dmag * np.abs(x) * r).sum((0, 1))
    turn = 8 * 2.0 ** -53 * np.abs(pos)[:, None, None]
    return y, mag * (32 * U32 + turn), dx, dxmag * (64 * U32 + turn), dg, dgmag * (256 * U32 + turn.max(initial=0))


def _close(got, ref, tol, what):
    half = {"bfloat16": 2.0 ** -8, "float32": 0.0}[str(got.dtype).split(".")[-1]]
    g = got.double().cpu().numpy()
    off = np.abs(g - ref) - (half * 1.001 * np.abs(ref) + tol)
    assert np.all(off <= 0), f"{what}: {off.max():.3e} over, at {np.unravel_index(off.argmax(), off.shape)}"


def _run(i, pos0, eps, theta=THETA, overwrite=True, dg0=None, stream=None):
    import torch
    from paper_2606_01143_amd import binding as B
    q, k = i["q"], i["k"]
    (T, hq, d), hkv = q.shape, k.shape[1]
    yq, yk = torch.empty(T, hq, d, dtype=q.dtype, device="cuda"), torch.empty(T, hkv, d, dtype=q.dtype, device="cuda")
    B.head_norm_rope_fwd(q, k, i["gq"], i["gk"], yq, yk, pos0, theta, positions=i["pos"], eps=eps, stream=stream)
    grad = torch.full_like(i["x"], 7.0) if T else torch.empty_like(i["x"])
    dq, dk = i["cut"](grad, 0, hq), i["cut"](grad, hq, hkv)
    dgq, dgk = (torch.full((d,), float("nan") if dg0 is None else dg0, device="cuda") for _ in range(2))
    ws = torch.empty(B.head_norm_rope_bwd_workspace_size(T, hq, hkv, d), dtype=torch.uint8, device="cuda")
    B.head_norm_rope_bwd(q, k, i["gq"], i["gk"], i["dyq"], i["dyk"], dq, dk, dgq, dgk, pos0, theta,
                         positions=i["pos"], eps=eps, overwrite=overwrite, ws=ws, stream=stream)
    torch.cuda.synchronize()
    return dict(yq=yq, yk=yk, dq=dq, dk=dk, dgq=dgq, dgk=dgk, grad=grad)


def _check(i, got, pos, eps, theta=THETA, dg0=0.0):
    for n in ("q", "k"):
        y, ty, dx, tx, dg, tg = _ref(i[n], i["g" + n], i["dy" + n], pos, eps, theta)
        _close(got["y" + n], y, ty, "y" + n)
        _close(got["d" + n], dx, tx, "d" + n)
        _close(got["dg" + n], dg + dg0, tg + abs(dg0) * U32, "dg" + n)


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


@pytest.mark.parametrize("T,hq,hkv,d,dt,extra,lead", [
    (1, 32, 4, 128, "bf16", 0, 0), (3, 5, 1, 128, "bf16", 0, 0), (67, 32, 8, 128, "bf16", 0, 0),
    (130, 4, 4, 64, "bf16", 64, 0), (33, 8, 2, 256, "bf16", 0, 0), (40, 6, 3, 96, "bf16", 0, 0),
    (9, 1, 1, 16, "bf16", 0, 0), (21, 3, 2, 80, "bf16", 0, 8),
    # rows and strides off 16 bytes, odd halves, the smallest head
    (21, 3, 2, 80, "bf16", 0, 1), (17, 3, 1, 72, "bf16", 3, 0), (50, 2, 2, 6, "bf16", 0, 0),
    (12, 2, 1, 250, "bf16", 0, 0), (300, 3, 1, 2, "bf16", 1, 1),
    (1, 32, 8, 128, "f32", 0, 0), (129, 8, 2, 64, "f32", 0, 0), (31, 4, 1, 256, "f32", 4, 0),
    (19, 2, 1, 72, "f32", 1, 0), (25, 20, 5, 112, "f32", 0, 0), (1025, 4, 2, 128, "bf16", 0, 0)])
def test_against_the_formulas(gpu, T, hq, hkv, d, dt, extra, lead):
    _say(f"T {T} heads {hq}/{hkv} d {d} {dt} extra {extra} lead {lead}")
    i = _inputs(T, hq, hkv, d, _dt(dt), seed=T + d, extra=extra, lead=lead)
    got = _run(i, 8191, 1e-6)
    _check(i, got, 8191.0 + np.arange(T), 1e-6)
    # the value heads between two tokens' keys and the padding stay as they were
    import torch
    rest = got["grad"][:, (hq + hkv) * d:]
    assert torch.equal(rest, torch.full_like(rest, 7.0))


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("bf16", 72), ("f32", 64), ("f32", 72)])
def test_small_rows_without_eps(gpu, dt, d):
    """Rows whose 1 / rms has a cube beyond fp32's range, but no gradient has."""
    i = _inputs(9, 3, 2, d, _dt(dt), seed=d)
    i["x"].mul_(2.0 ** -48)
    _check(i, _run(i, 5, 0.0), 5 + np.arange(9), 0.0)


def test_more_rows_than_a_launch_has_waves(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    T = (1 << 24) + 5
    _say(f"T {T} heads 1/1 d 2")
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    q, k, gq, gk = r(T, 1, 2), r(T, 1, 2), r(2), r(2)
    yq, yk = torch.zeros_like(q), torch.zeros_like(k)
    B.head_norm_rope_fwd(q, k, gq, gk, yq, yk, 0, THETA)
    for at in (slice(0, 5), slice(T // 2, T // 2 + 9), slice(T - 30, T)):
        pos = np.arange(at.start, at.stop, dtype=np.float64)
        for x, gain, y in ((q, gq, yq), (k, gk, yk)):
            ref, tol = _ref(x[at], gain, x[at], pos, 1e-6)[:2]
            _close(y[at], ref, tol, f"y at {at}")


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f32", 64), ("bf16", 72)])
def test_positions(gpu, dt, d):
    """Packed suffixes, a repeated and a negative position, and far ones."""
    pos = [0, 1, 2, 0, 1, 5, 5, -3, 100000, 16777217, 2147483647, -2147483648]
    i = _inputs(len(pos), 4, 2, d, _dt(dt), seed=5, positions=pos)
    _check(i, _run(i, 4096, 1e-5), np.array(pos, dtype=np.float64) + 4096, 1e-5)
    i = _inputs(len(pos), 4, 2, d, _dt(dt), seed=6, positions=pos)
    _check(i, _run(i, 0, 1e-5, theta=10000.0), np.array(pos, dtype=np.float64), 1e-5, theta=10000.0)


def test_gain_gradient_sums_and_repeats(gpu):
    """Added to what is there, over many rows, bitwise the same twice."""
    import torch
    i = _inputs(700, 8, 2, 128, torch.bfloat16, seed=8)
    a, b = _run(i, 0, 1e-6, overwrite=False, dg0=3.0), _run(i, 0, 1e-6, overwrite=False, dg0=3.0)
    _check(i, a, np.arange(700.0), 1e-6, dg0=3.0)
    assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_gradients_against_differences(gpu, dt):
    """The 64-bit formula that the other tests hold the kernels to has the
    derivatives of its own forward."""
    i = _inputs(3, 2, 1, 6, _dt(dt), seed=11)
    x, g, dy = (i[n].double().cpu().numpy() for n in ("q", "gq", "dyq"))
    pos = np.array([3.0, 9.0, 4.0])

    def loss(x, g):
        import torch
        t = lambda v: torch.from_numpy(v)
        return (_ref(t(x), t(g), t(dy), pos, 1e-5)[0] * dy).sum()
    _, _, dx, _, dg, _ = _ref(i["q"], i["gq"], i["dyq"], pos, 1e-5)
    e = 1e-6
    for at in [(0, 0, 0), (1, 1, 5), (2, 0, 3)]:
        step = np.zeros_like(x)
        step[at] = e
        assert abs((loss(x + step, g) - loss(x - step, g)) / (2 * e) - dx[at]) < 1e-7 * (1 + abs(dx[at])) * 100
    for j in range(6):
        step = np.zeros_like(g)
        step[j] = e
        assert abs((loss(x, g + step) - loss(x, g - step)) / (2 * e) - dg[j]) < 1e-7 * (1 + abs(dg[j])) * 100


@pytest.mark.parametrize("d", [128, 72])
def test_a_bad_row_stays_in_its_row(gpu, d):
    import torch
    i = _inputs(70, 4, 2, d, torch.bfloat16, seed=9)
    clean = _run(i, 0, 1e-6)
    i["x"][33, 2 * d + 5] = float("nan")   # q head 2 of token 33
    i["x"][40, 5 * d + 1] = float("inf")   # k head 1 of token 40
    got = _run(i, 0, 1e-6)
    for n, t, h in (("q", 33, 2), ("k", 40, 1)):
        for w in ("y", "d"):
            a, b = got[w + n].clone(), clean[w + n].clone()
            assert not torch.isfinite(a[t, h]).all()
            a[t, h] = b[t, h] = 0
            assert torch.equal(a, b), w + n
    # an all-zero row: finite at eps > 0, y = 0
    i = _inputs(5, 2, 1, d, torch.bfloat16, seed=10)
    i["x"][2] = 0
    got = _run(i, 0, 1e-6)
    assert got["yq"][2].abs().max() == 0 and torch.isfinite(got["dq"]).all()
    _check(i, got, np.arange(5.0), 1e-6)


def test_no_tokens(gpu):
    import torch
    i = _inputs(0, 4, 2, 128, torch.bfloat16, seed=1)
    got = _run(i, 0, 1e-6)
    assert got["dgq"].abs().max() == 0 and got["dgk"].abs().max() == 0
    got = _run(i, 0, 1e-6, overwrite=False, dg0=2.0)
    assert torch.equal(got["dgq"], torch.full((128,), 2.0, device="cuda"))


def test_captured_and_on_another_stream(gpu):
    """Two captured graphs with a workspace each, replayed several times with
    eager work between, and an explicit stream."""
    import torch
    from paper_2606_01143_amd import binding as B
    _say("graph")
    ins = [_inputs(T, 8, 2, 128, torch.bfloat16, seed=T) for T in (64, 200)]
    eager = [_run(i, 5, 1e-6) for i in ins]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _run(ins[1], 5, 1e-6, stream=side)
    assert all(torch.equal(got[n], eager[1][n]) for n in got)
    caught = []
    for i in ins:
        (T, hq, d), hkv = i["q"].shape, 2
        o = dict(yq=torch.empty_like(i["dyq"]), yk=torch.empty_like(i["dyk"]), dq=torch.empty_like(i["dyq"]),
                 dk=torch.empty_like(i["dyk"]), dgq=torch.empty(d, device="cuda"), dgk=torch.empty(d, device="cuda"),
                 ws=torch.empty(B.head_norm_rope_bwd_workspace_size(T, hq, hkv, d), dtype=torch.uint8, device="cuda"))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.head_norm_rope_fwd(i["q"], i["k"], i["gq"], i["gk"], o["yq"], o["yk"], 5, THETA, eps=1e-6)
            B.head_norm_rope_bwd(i["q"], i["k"], i["gq"], i["gk"], i["dyq"], i["dyk"], o["dq"], o["dk"], o["dgq"],
                                 o["dgk"], 5, THETA, eps=1e-6, overwrite=True, ws=o["ws"])
        caught.append((graph, o))
    for _ in range(4):
        for (graph, o), e in zip(caught, eager):
            for t in o.values():
                t.fill_(1)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o[n], e[n]) for n in o if n != "ws")
            _run(ins[0], 5, 1e-6)


@pytest.mark.parametrize("d,stride", [(128, (1 << 30) + 8), (72, (1 << 30) + 9)])
def test_far_strides(gpu, d, stride):
    """Three tokens more than 2^30 elements apart give what contiguous ones give."""
    import torch
    from paper_2606_01143_amd import binding as B
    _say(f"stride {stride} d {d}")
    i = _inputs(3, 4, 2, d, torch.bfloat16, seed=d)
    want = _run(i, 9, 1e-6)
    buf = torch.empty(2 * stride + 6 * d, dtype=torch.bfloat16, device="cuda")
    view = lambda b, a, n: b[a * d:].as_strided((3, n, d), (stride, d, 1))
    q, k = view(buf, 0, 4), view(buf, 4, 2)
    q.copy_(i["q"])
    k.copy_(i["k"])
    yq, yk = torch.empty_like(i["dyq"]), torch.empty_like(i["dyk"])
    B.head_norm_rope_fwd(q, k, i["gq"], i["gk"], yq, yk, 9, THETA)
    grad = torch.empty_like(buf)
    dq, dk = view(grad, 0, 4), view(grad, 4, 2)
    dgq, dgk = (torch.empty(d, device="cuda") for _ in range(2))
    ws = torch.empty(B.head_norm_rope_bwd_workspace_size(3, 4, 2, d), dtype=torch.uint8, device="cuda")
    B.head_norm_rope_bwd(q, k, i["gq"], i["gk"], i["dyq"], i["dyk"], dq, dk, dgq, dgk, 9, THETA, overwrite=True, ws=ws)
    got = dict(yq=yq, yk=yk, dq=dq, dk=dk, dgq=dgq, dgk=dgk)
    if d == 128:  # the same kernel: both take 16-byte chunks
        assert all(torch.equal(t, want[n]) for n, t in got.items())
    _check(i, got, 9 + np.arange(3.0), 1e-6)
