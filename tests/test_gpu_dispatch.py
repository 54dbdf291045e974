"""The plan against a stable sort, the weighted sum and its backward against
the formulas in 64 bits, and a layer of experts run from the router's choices
to its gradients.

A weighted sum of k bf16 values adds k products and the residual in fp32
(2^-24 of the magnitudes each) and is rounded once (2^-8); a dot product of
`width` terms is off by at most 2^-24 of the magnitudes a term."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
HALF = 2.0 ** -8 * 1.001


def _say(what):
    print(f"\n[gpu dispatch] {what}", flush=True)


def _plan(E, ids):
    import torch
    from paper_2606_01143_amd import binding as B
    T, k = ids.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    out = [torch.full((E + 1,), 77, **i32), torch.full((T * k,), 77, **i32), torch.full((T, k), 77, **i32)]
    ws = torch.empty(B.experts_plan_workspace_size(E, k, T), dtype=torch.uint8, device="cuda")
    B.experts_plan(E, ids, *out, ws=ws)
    return out


def _want(E, ids):
    flat = ids.reshape(-1)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    counts = np.bincount(key, minlength=E + 1)[:E]
    offsets = np.concatenate([[0], np.cumsum(counts)])
    n = offsets[-1]
    row_token = np.where(np.arange(flat.size) < n, order // ids.shape[1], -1)
    pos = np.empty(flat.size, dtype=np.int64)
    pos[order] = np.arange(flat.size)
    return offsets, row_token, np.where(key < E, pos, -1).reshape(ids.shape)


@pytest.mark.parametrize("T,k,E,kind", [
    (1, 1, 1, "any"), (1, 8, 128, "any"), (4, 8, 128, "any"), (63, 3, 5, "any"), (129, 8, 8, "any"),
    (1000, 2, 1024, "any"), (8192, 8, 128, "any"), (3001, 4, 60, "padded"), (257, 6, 64, "dropped"),
    (500, 8, 256, "one"), (70001, 1, 7, "padded"), (20000, 8, 1023, "padded"), (40, 2, 3, "twice"), (0, 4, 16, "any"),
    (512, 8, 128, "any"), (513, 8, 128, "any"), (1024, 1, 2, "any"),
    # either side of the count in a launch of its own
    (4096, 1, 1024, "padded"), (4097, 1, 1024, "padded"), (2049, 2, 2, "any")])
def test_plan(gpu, T, k, E, kind):
    import torch
    _say(f"T {T} k {k} E {E} {kind}")
    rng = np.random.default_rng(T + E)
    ids = rng.integers(0, E, (T, k))
    if kind == "padded":
        ids[rng.random((T, k)) < 0.3] = rng.choice(np.array([-1, E, 2147483647, -2147483648]))
        ids[: T // 4] = -1
    elif kind == "dropped":
        ids[:] = -1
    elif kind == "one":
        ids[:] = E - 1
    elif kind == "twice":
        ids[:, 1] = ids[:, 0]
    got = _plan(E, torch.from_numpy(ids).to(torch.int32).cuda())
    for g, w, n in zip(got, _want(E, ids), ("offsets", "row_token", "pos")):
        assert np.array_equal(g.cpu().numpy(), w), n


@pytest.mark.parametrize("T,k,width,drop", [(1, 1, 8, 0.0), (1, 8, 2048, 0.0), (7, 3, 40, 0.5), (130, 8, 520, 0.2),
                                            (33, 1, 4096, 0.0), (65, 12, 2056, 1.0), (300, 6, 136, 0.3),
                                            (5, 1024, 16, 0.1)])
@pytest.mark.parametrize("weighted,added", [(True, True), (False, False), (True, False)])
def test_combine(gpu, T, k, width, drop, weighted, added):
    import torch
    from paper_2606_01143_amd import binding as B
    _say(f"T {T} k {k} width {width} drop {drop}")
    rng = np.random.default_rng(T + width)
    R = T * k
    pos = rng.permutation(R).reshape(T, k)
    pos[rng.random((T, k)) < drop] = rng.choice(np.array([-1, R, 2147483647]))
    kept = torch.from_numpy((pos >= 0) & (pos < R)).cuda()
    at = torch.from_numpy(np.where((pos >= 0) & (pos < R), pos, 0)).cuda()
    p = torch.from_numpy(pos).to(torch.int32).cuda()
    g = torch.Generator(device="cuda").manual_seed(width)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    y, dout, res = r(R, width).bfloat16(), r(T, width).bfloat16(), r(T, width).bfloat16()
    w = r(T, k) if weighted else None
    wd = torch.where(kept, w.double() if weighted else 1.0, 0.0)
    out = res.clone() if added else torch.empty_like(res)
    B.experts_combine_fwd(y, p, w, out, add=out if added else None)   # in place where added
    terms = wd[..., None] * torch.where(kept[..., None], y[at].double(), 0.0)
    ref, mag = terms.sum(1), terms.abs().sum(1)
    if added:
        ref, mag = ref + res.double(), mag + res.double().abs()
    assert ((out.double() - ref).abs() <= HALF * ref.abs() + (2 * k + 1) * U32 * mag).all()
    dy, dw = torch.full_like(y, 3.0), torch.full((T, k), 3.0, device="cuda")
    B.experts_combine_bwd(dout, y, p, w, dy, dw)
    want = torch.full(y.shape, 3.0, dtype=torch.float64, device="cuda")
    want[at[kept]] = (wd[..., None] * dout.double()[:, None])[kept]
    assert ((dy.double() - want).abs() <= HALF * want.abs()).all()
    prod = torch.where(kept[..., None], y[at].double(), 0.0) * dout.double()[:, None]
    assert ((dw.double() - prod.sum(-1)).abs() <= (width + 1) * U32 * prod.abs().sum(-1)).all()
    only = torch.full_like(y, 3.0)
    B.experts_combine_bwd(dout, None, p, w, only, None)
    assert torch.equal(only, dy)


def test_combine_ignores_skipped_rows_values(gpu):
    """A dropped choice's weight may be anything, and NaN rows that no choice
    names reach nothing."""
    import torch
    from paper_2606_01143_amd import binding as B
    y = torch.ones(6, 16, device="cuda").bfloat16()
    y[3:] = float("nan")
    pos = torch.tensor([[0, -1], [1, 2]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[2.0, float("nan")], [3.0, float("inf")]], device="cuda")
    out = torch.empty(2, 16, device="cuda").bfloat16()
    B.experts_combine_fwd(y, pos, w, out)
    assert (out[0] == 2).all() and out[1].isinf().all()
    dy, dw = torch.zeros_like(y), torch.empty(2, 2, device="cuda")
    B.experts_combine_bwd(out, y, pos, w, dy, dw)
    assert dw[0, 0] == 32 and dw[0, 1] == 0 and (dy[3:] == 0).all()


def test_more_choices_than_a_launch_has_waves(gpu):
    """Small whole numbers: every sum and rounding is exact."""
    import torch
    from paper_2606_01143_amd import binding as B
    T, k, width = (1 << 23) + 7, 4, 8
    R = T * k
    _say(f"combine T {T} k {k} width {width}")
    g = torch.Generator(device="cuda").manual_seed(1)
    whole = lambda *s: torch.randint(-8, 9, s, generator=g, device="cuda", dtype=torch.int8)
    y, dout, w = whole(R, width).bfloat16(), whole(T, width).bfloat16(), whole(T, k).float() / 2
    pos = torch.arange(R - 1, -1, -1, dtype=torch.int32, device="cuda").view(T, k)
    out = torch.empty(T, width, dtype=torch.bfloat16, device="cuda")
    B.experts_combine_fwd(y, pos, w, out)
    mine = y.flip(0).view(T, k, width)
    assert torch.equal(out, (w[..., None] * mine).sum(1).bfloat16())
    dy, dw = torch.empty_like(y), torch.empty_like(w)
    B.experts_combine_bwd(dout, y, pos, w, dy, dw)
    assert torch.equal(dw, (mine.float() * dout.float()[:, None]).sum(-1))
    assert torch.equal(dy.flip(0).view(T, k, width), (w[..., None] * dout[:, None]).bfloat16())


def test_no_tokens(gpu):
    import torch
    from paper_2606_01143_amd import binding as B
    bf = dict(dtype=torch.bfloat16, device="cuda")
    y, pos = torch.empty(0, 16, **bf), torch.empty(0, 4, dtype=torch.int32, device="cuda")
    w = torch.empty(0, 4, device="cuda")
    B.experts_combine_fwd(y, pos, w, torch.empty(0, 16, **bf))
    B.experts_combine_bwd(torch.empty(0, 16, **bf), y, pos, w, torch.empty(0, 16, **bf), torch.empty(0, 4, device="cuda"))


# ------------------------------------------------ a layer, as it would be used
class Layer:
    """norm -> router's given choices -> experts -> residual, and its backward,
    in the call order of a trainer."""

    def __init__(self, T, E, k, h, inter, seed, padded):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s, sc=1.0: (torch.randn(*s, generator=g, device="cuda") * sc).bfloat16()
        self.E, self.x, self.dout = E, r(T, h), r(T, h)
        self.wg, self.wu, self.wd = r(E, h, inter, sc=0.1), r(E, h, inter, sc=0.1), r(E, inter, h, sc=0.1)
        self.ids = torch.rand(T, E, generator=g, device="cuda").topk(k, 1).indices.to(torch.int32)
        self.p = torch.rand(T, k, generator=g, device="cuda")
        if padded:
            self.ids[-padded:] = -1

    def run(self, dw=None):
        import torch
        from paper_2606_01143_amd import binding as B
        T, h = self.x.shape
        k, E, inter = self.ids.shape[1], self.E, self.wg.shape[2]
        R = T * k
        i32, bf = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
        off, tok, pos = torch.empty(E + 1, **i32), torch.empty(R, **i32), torch.empty(T, k, **i32)
        ws = torch.empty(B.experts_plan_workspace_size(E, k, T), dtype=torch.uint8, device="cuda")
        B.experts_plan(E, self.ids, off, tok, pos, ws=ws)
        # rows that are nobody's hold zeros: SwiGLU runs over them too
        gt, up, m = (torch.zeros(R, inter, **bf) for _ in range(3))
        y, out = torch.empty(R, h, **bf), torch.empty(T, h, **bf)
        B.experts_fwd(off, self.x, self.wg, gt, w2=self.wu, y2=up, row_token=tok)
        B.swiglu_fwd(gt, up, m)
        B.experts_fwd(off, m, self.wd, y)
        B.experts_combine_fwd(y, pos, self.p, out, add=self.x)
        dy, dp = torch.zeros(R, h, **bf), torch.empty(T, k, device="cuda")
        B.experts_combine_bwd(self.dout, y, pos, self.p, dy, dp)
        first = dw is None
        if first:
            dw = [torch.empty(w.shape, device="cuda") for w in (self.wg, self.wu, self.wd)]
        dm, dg, du = (torch.zeros(R, inter, **bf) for _ in range(3))
        B.experts_bwd_w(off, m, dy, dw[2], overwrite=first)
        B.experts_bwd_x(off, dy, self.wd, dm)
        B.swiglu_bwd(gt, up, dm, dg, du)
        B.experts_bwd_w(off, self.x, dg, dw[0], dy2=du, dw2=dw[1], row_token=tok, overwrite=first)
        dxr, dx = torch.empty(R, h, **bf), torch.empty(T, h, **bf)
        B.experts_bwd_x(off, dg, self.wg, dxr, dy2=du, w2=self.wu)
        B.experts_combine_fwd(dxr, pos, None, dx, add=self.dout)
        return dict(out=out, dx=dx, dp=dp, dwg=dw[0], dwu=dw[1], dwd=dw[2])

    def reference(self):
        """The same layer token by token in 64 bits, gradients by autograd on the CPU."""
        import torch
        c = lambda t: t.double().cpu().requires_grad_()
        x, wg, wu, wd, p = c(self.x), c(self.wg), c(self.wu), c(self.wd), c(self.p)
        ids, out = self.ids.cpu().long(), []
        for t in range(x.shape[0]):
            o = x[t]
            for j in range(ids.shape[1]):
                e = ids[t, j]
                if e >= 0:
                    o = o + p[t, j] * ((torch.nn.functional.silu(x[t] @ wg[e]) * (x[t] @ wu[e])) @ wd[e])
            out.append(o)
        out = torch.stack(out)
        (out * self.dout.double().cpu()).sum().backward()
        return dict(out=out.detach(), dx=x.grad, dp=p.grad, dwg=wg.grad, dwu=wu.grad, dwd=wd.grad)


@pytest.mark.parametrize("T,E,k,h,inter,padded", [(70, 8, 2, 64, 96, 0), (41, 16, 4, 136, 72, 9), (1, 6, 3, 64, 64, 0)])
def test_a_layer_of_experts(gpu, T, E, k, h, inter, padded):
    """Every tensor kept between the calls is rounded to bf16 once (2^-8); a
    result lies behind at most six such tensors, so that max-abs-relative
    errors stay under 6 x 2^-8 = 2.4e-2; the weights' gradients and the
    router's likewise."""
    _say(f"layer T {T} E {E} k {k} h {h} inter {inter}")
    layer = Layer(T, E, k, h, inter, seed=T, padded=padded)
    got, ref = layer.run(), layer.reference()
    for n, r in ref.items():
        err = (got[n].double().cpu() - r).abs().max() / r.abs().max()
        assert err <= 6 * 2.0 ** -8, (n, err.item())
    if padded:
        import torch
        assert torch.equal(got["out"][-padded:], layer.x[-padded:]) and not got["dp"][-padded:].any()


def test_prefix_part_and_suffix_parts_add_up(gpu):
    """Weight gradients of two token sets into one sum, bitwise repeatable."""
    import torch
    a, b = Layer(60, 8, 2, 64, 64, 1, 0), Layer(23, 8, 2, 64, 64, 2, 5)
    b.wg, b.wu, b.wd = a.wg, a.wu, a.wd
    keys = ("dwg", "dwu", "dwd")
    runs = []
    for _ in range(2):
        first = a.run()
        alone = [first[n].clone() for n in keys]
        both = b.run(dw=[first[n] for n in keys])
        runs.append([both[n] for n in keys])
    own = b.run()
    for s, x, n in zip(runs[0], alone, keys):
        ref = x.double() + own[n].double()
        off = (s.double() - ref).abs() - (40 * U32 * (x.abs() + own[n].abs()).double() + 1e-6)
        assert off.max().item() <= 0, n
    assert all(torch.equal(x, y) for x, y in zip(*runs))


def test_layer_captured(gpu):
    import torch
    _say("graph")
    layers = [Layer(50, 8, 2, 64, 64, 3, 6), Layer(4, 16, 4, 64, 64, 4, 0)]
    eager = [layer.run() for layer in layers]
    graphs = []
    for layer in layers:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = layer.run()
        graphs.append((graph, out))
    for _ in range(4):
        for (graph, out), e, layer in zip(graphs, eager, layers):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[n], e[n]) for n in e)
            layer.run()
