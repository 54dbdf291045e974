"""Embedding lookup and its gradient against the formulas in 64 bits.

A forward value is one fp32 product rounded to its type (half a step of each).
A gradient element adds its token's count of terms and the table's value in
fp32: each addition is off by at most 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


def _say(what):
    print(f"\n[gpu embed] {what}", flush=True)


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _ids(kind, T, V, seed):
    rng = np.random.default_rng(seed)
    if kind == "any":
        return rng.integers(0, V, T)
    if kind == "few":       # long runs of few ids
        return rng.choice(np.array([0, V // 2, V - 1]), T)
    if kind == "one":
        return np.full(T, V - 1)
    if kind == "frequent":  # as text: the logarithm is uniform
        return np.clip(np.exp(rng.uniform(0, np.log(V + 1), T)).astype(np.int64) - 1, 0, V - 1)
    if kind == "padded":    # ids outside the table on both sides among them
        ids = rng.integers(0, V, T)
        ids[rng.random(T) < 0.4] = -1
        ids[rng.random(T) < 0.1] = V
        ids[rng.random(T) < 0.1] = 2147483647
        ids[rng.random(T) < 0.1] = -2147483648
        return ids
    if kind == "dropped":
        return np.full(T, -1)
    raise KeyError(kind)


def _bwd(ids, dy, table, scale, **kw):
    import torch
    from paper_2606_01143_amd import binding as B
    ws = torch.empty(B.embed_bwd_workspace_size(dy.shape[0], table.shape[0], table.shape[1]), dtype=torch.uint8,
                     device="cuda")
    B.embed_bwd(ids, dy, table, scale=scale, ws=ws, **kw)


CASES = [(1, 7, 8, "any", "bf16"), (5, 1, 64, "one", "f32"), (64, 100, 520, "any", "bf16"),
         (333, 1000, 136, "frequent", "f32"), (1000, 3, 64, "any", "bf16"), (257, 513, 24, "padded", "bf16"),
         (4097, 128000, 64, "frequent", "bf16"), (1024, 511, 40, "any", "f32"), (2000, 40, 72, "one", "bf16"),
         (3000, 262144, 16, "few", "f32"), (129, 65, 4096, "padded", "f32"), (50, 9, 16, "dropped", "bf16"),
         (20011, 50000, 8, "frequent", "f32"), (70001, 300, 8, "any", "bf16"), (2049, 2147483, 8, "any", "bf16"),
         # either side of the count in a launch of its own, and many spans of one id
         (4096, 700, 8, "frequent", "f32"), (65537, 700, 8, "frequent", "f32"), (33, 5, 8, "one", "bf16"),
         (32, 5, 8, "few", "f32"), (40000, 100, 72, "padded", "bf16"),
         (8192, 900, 8, "frequent", "bf16"), (8191, 128000, 8, "any", "f32"), (8190, 50, 24, "padded", "bf16"),
         (8193, 900, 8, "frequent", "f32"), (5000, 6, 8, "one", "bf16"), (7777, 7, 8, "dropped", "f32"),
         # the direct form's last size, ranks by counting up to theirs, and a row's ids in any part
         (256, 40, 520, "padded", "bf16"), (256, 3, 8, "one", "f32"), (255, 200, 1032, "any", "f32"),
         (257, 20, 520, "frequent", "bf16"), (4095, 2147483, 8, "padded", "f32"), (4097, 50, 24, "few", "bf16")]


@pytest.mark.parametrize("T,V,width,kind,dt", CASES)
def test_against_the_formulas(gpu, T, V, width, kind, dt):
    import torch
    from paper_2606_01143_amd import binding as B
    _say(f"T {T} V {V} width {width} {kind} {dt}")
    ids = _ids(kind, T, V, seed=T)
    g = torch.Generator(device="cuda").manual_seed(T + V)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    table, dy, grad = rnd(V, width).to(_dt(dt)), rnd(T, width).to(_dt(dt)), rnd(V, width)
    dev = torch.from_numpy(ids.astype(np.int64)).to(torch.int32).cuda()
    scale = float(np.float32(1.7))
    valid = (ids >= 0) & (ids < V)
    y = torch.full((T, width), float("nan"), dtype=table.dtype, device="cuda")
    B.embed_fwd(dev, table, y, scale=scale)
    at = torch.from_numpy(np.where(valid, ids, 0)).cuda()
    ref = torch.where(torch.from_numpy(valid).cuda()[:, None], table[at].double() * scale, 0.0)
    half = {"bf16": 2.0 ** -8, "f32": 0.0}[dt]
    assert ((y.double() - ref).abs() <= (half * 1.001 + 2 * U32) * ref.abs()).all()
    before = grad.clone()
    _bwd(dev, dy, grad, scale)
    kept, rows = dy.double()[torch.from_numpy(valid).cuda()], at[torch.from_numpy(valid).cuda()]
    want = before.double().index_add_(0, rows, kept * scale)
    mag = before.double().abs().index_add_(0, rows, kept.abs() * scale)
    count = torch.zeros(V, device="cuda", dtype=torch.float64).index_add_(0, rows, torch.ones_like(rows).double())
    tol = (count[:, None] + 4) * U32 * mag
    off = (grad.double() - want).abs() - tol
    assert (off <= 0).all(), off.max().item()
    untouched = count == 0
    assert torch.equal(grad[untouched], before[untouched])


def test_gradient_repeats_and_adds_parts(gpu):
    """Bitwise the same twice, and the prefix's part then the suffixes'."""
    import torch
    ids = torch.from_numpy(_ids("frequent", 5000, 900, 3)).to(torch.int32).cuda()
    dy = torch.randn(5000, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    runs = []
    for _ in range(2):
        t = torch.zeros(900, 256, device="cuda")
        _bwd(ids[:3000], dy[:3000], t, 2.0)
        _bwd(ids[3000:].clone(), dy[3000:], t, 2.0)
        runs.append(t)
    assert torch.equal(runs[0], runs[1])
    want = torch.zeros(900, 256, device="cuda", dtype=torch.float64).index_add_(0, ids.long(), dy.double() * 2)
    assert (runs[0].double() - want).abs().max() <= 1e-4 * want.abs().max()


def test_gradient_is_the_forwards_derivative(gpu):
    """<dy, lookup(table)> = <gradient, table> for a linear lookup, in 64 bits."""
    import torch
    from paper_2606_01143_amd import binding as B
    ids = torch.from_numpy(_ids("padded", 400, 60, 5)).to(torch.int32).cuda()
    g = torch.Generator(device="cuda").manual_seed(2)
    table, dy = (torch.randn(n, 64, generator=g, device="cuda") for n in (60, 400))
    y, grad = torch.empty(400, 64, device="cuda"), torch.zeros(60, 64, device="cuda")
    B.embed_fwd(ids, table, y, scale=0.5)
    _bwd(ids, dy, grad, 0.5)
    a, b = (y.double() * dy.double()).sum(), (grad.double() * table.double()).sum()
    # 400 x 64 products, at most 400 fp32 additions deep each
    bound = 404 * U32 * (y.double() * dy.double()).abs().sum()
    assert (a - b).abs() <= bound


def test_a_bad_row_reaches_its_own_id(gpu):
    import torch
    ids = torch.tensor([4, 2, 4, 9, 2, -1], dtype=torch.int32, device="cuda")
    dy = torch.ones(6, 8, device="cuda")
    dy[2] = float("nan")
    dy[5] = float("inf")
    t = torch.zeros(10, 8, device="cuda")
    _bwd(ids, dy, t, 1.0)
    assert t[4].isnan().all() and t[2].eq(2).all() and t[9].eq(1).all()
    t[4] = 0
    assert t.sum() == 24


def test_more_values_than_a_launch_has_threads_for(gpu):
    """An output of 34 GB."""
    import torch
    from paper_2606_01143_amd import binding as B
    T, width = (1 << 18) + 3, 65536
    _say(f"fwd T {T} width {width}")
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    g = torch.Generator(device="cuda").manual_seed(5)
    table = torch.randn(4, width, generator=g, device="cuda").bfloat16()
    ids = torch.randint(-1, 4, (T,), generator=g, device="cuda", dtype=torch.int32)
    y = torch.empty(T, width, dtype=torch.bfloat16, device="cuda")
    B.embed_fwd(ids, table, y, scale=0.5)   # a power of two: no rounding
    padded = torch.cat([table * 0.5, torch.zeros_like(table[:1])])
    for at in range(0, T, 1 << 13):
        part = y[at:at + (1 << 13)]
        assert torch.equal(part, padded[ids[at:at + (1 << 13)].long()]), f"rows {at} on"
    del y, part
    torch.cuda.empty_cache()


def test_no_tokens(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    t = torch.ones(5, 8, device="cuda")
    B.embed_fwd(ids, t, torch.empty(0, 8, device="cuda"))
    assert B.embed_bwd_workspace_size(0, 5, 8) == 0
    B.embed_bwd(ids, torch.empty(0, 8, device="cuda"), t)
    assert t.eq(1).all()


def test_captured_and_on_another_stream(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    _say("graph")
    side = torch.cuda.Stream()
    parts = []
    for T, V in ((300, 50), (4000, 70000)):
        ids = torch.from_numpy(_ids("frequent", T, V, T)).to(torch.int32).cuda()
        dy = torch.randn(T, 128, device="cuda").bfloat16()
        eager = torch.zeros(V, 128, device="cuda")
        _bwd(ids, dy, eager, 1.5)
        other = torch.zeros(V, 128, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        _bwd(ids, dy, other, 1.5, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(eager, other)
        ws = torch.empty(B.embed_bwd_workspace_size(T, V, 128), dtype=torch.uint8, device="cuda")
        graph, t = torch.cuda.CUDAGraph(), torch.zeros(V, 128, device="cuda")
        with torch.cuda.graph(graph):
            B.embed_bwd(ids, dy, t, scale=1.5, ws=ws)
        parts.append((graph, t, ws, eager, ids, dy))  # a graph's inputs stay alive
    for _ in range(4):
        for graph, t, ws, eager, *_ in parts:
            t.zero_()
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(t, eager)
            (eager * 2).sum()


def test_few_tokens_of_more_columns_than_a_launch_has_waves(gpu):
    """256 tokens by 2^27 + 520 columns: a wave for a token and 512 columns would be
    more than 2^32 threads.  Whole numbers, which fp32 adds exactly."""
    import torch
    T, V, width = 256, 2, (1 << 27) + 520
    _say(f"bwd T {T} width {width}")
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    g = torch.Generator(device="cuda").manual_seed(7)
    row = torch.randint(-4, 5, (width,), generator=g, device="cuda").bfloat16()
    times = torch.randint(-3, 4, (T,), generator=g, device="cuda").bfloat16()
    ids = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dy = torch.mul(times[:, None], row)
    table = torch.ones(V, width, device="cuda")
    _bwd(ids, dy, table, 0.5)
    for v in range(V):
        want = row.float() * (0.5 * times[ids == v].float().sum()) + 1
        assert torch.equal(table[v], want), f"row {v}"
    del dy, table, want
    torch.cuda.empty_cache()
