"""A decoder layer whose queries and keys are normalised per head, through the
schedule and dense, against the same layer in 64 bits with gradients by
autograd; the gate is the other layers' (max-abs-relative 2e-2 in bf16).  The
gains' gradients are the prefix part plus every suffix part."""
import numpy as np
import pytest
import torch

from oracle.compare import max_abs_rel
from oracle.layer import _tail, attention, rms, rope
from synthetic.layer import LayerShape, make_layer_group

TOL = 2e-2
KEYS = ("wq", "wk", "wv", "wo", "wg", "wu", "wd", "gq", "gk")


def _group(shape, seed):
    inp = make_layer_group(shape, seed=seed)
    rng = np.random.default_rng(seed)
    for k in ("gq", "gk"):
        g = torch.from_numpy(1 + 0.3 * rng.standard_normal(shape.head_dim)).bfloat16()
        inp["weights"] = dict(inp["weights"], **{k: g.float().numpy()})
    return inp


def _reference(inp):
    shp = inp["shape"]
    t64 = lambda x, grad=False: torch.tensor(np.asarray(x, dtype=np.float64), requires_grad=grad)
    W = {k: t64(inp["weights"][k], True) for k in KEYS}
    P, hq, hkv, d = shp.prefix_len, shp.num_q_heads, shp.num_kv_heads, shp.head_dim
    y_s, dx_s, dx_p, y_p = [], [], 0, None
    for x_s, dy_s, dy_p in zip(inp["x_s"], inp["dy_s"], inp["dy_p"]):
        x = t64(np.concatenate([inp["x_p"], x_s]), True)
        L = x.shape[0]
        n, pos = rms(x, shp.norm_eps), torch.arange(L)
        head = lambda w, g, h: rope(rms((n @ W[w]).view(L, h, d), shp.norm_eps) * W[g], pos, shp.rope_theta)
        o = attention(head("wq", "gq", hq), head("wk", "gk", hkv), (n @ W["wv"]).view(L, hkv, d),
                      torch.tril(torch.ones(L, L, dtype=torch.bool)))
        y = _tail(x, o, W, shp)
        y.backward(t64(np.concatenate([dy_p, dy_s])))
        dx_p = dx_p + x.grad[:P].numpy()
        dx_s.append(x.grad[P:].numpy())
        y_s.append(y[P:].detach().numpy())
        y_p = y[:P].detach().numpy()
    return {"y_p": y_p, "y_s": y_s, "dx_p": dx_p, "dx_s": dx_s, "dw": {k: W[k].grad.numpy() for k in KEYS}}


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [LayerShape(256, 4, 2, 64, 512, 200, (70, 33, 1)),
                                   LayerShape(512, 8, 2, 128, 256, 65, (130,))], ids=["d64", "d128"])
def test_schedule_and_dense(gpu, shape):
    from paper_2606_01143_amd.layer import DecoderLayer
    print(f"\n[gpu layer head norm] {shape}", flush=True)
    inp = _group(shape, seed=4)
    ref, layer = _reference(inp), DecoderLayer(inp)
    for got in (layer.run_schedule(), layer.run_dense()):
        errs = {"y_p": max_abs_rel(_np(got["y_p"]), ref["y_p"]), "dx_p": max_abs_rel(_np(got["dx_p"]), ref["dx_p"])}
        for i in range(shape.n):
            errs[f"y_s{i}"] = max_abs_rel(_np(got["y_s"][i]), ref["y_s"][i])
            errs[f"dx_s{i}"] = max_abs_rel(_np(got["dx_s"][i]), ref["dx_s"][i])
        errs.update({"d" + k: max_abs_rel(_np(got["dw"][k]), ref["dw"][k]) for k in KEYS})
        assert not {k: v for k, v in errs.items() if not v <= TOL}, errs


def test_gains_go_together():
    from paper_2606_01143_amd.layer import DecoderLayer
    inp = _group(LayerShape(64, 2, 1, 64, 64, 8, (4,)), seed=1)
    del inp["weights"]["gk"]
    with pytest.raises(ValueError, match="go together"):
        DecoderLayer(inp, device="cpu")


@pytest.mark.gpu
def test_from_the_embedding_and_back(gpu):
    """Token ids -> embedding -> the layer's schedule -> the table's gradient, the
    prefix's part once plus every suffix's.  A row of it adds its tokens' dx, each
    within the layer's gate of its part's largest."""
    from paper_2606_01143_amd import binding as B
    from paper_2606_01143_amd.layer import DecoderLayer
    shape, V = LayerShape(256, 4, 2, 64, 512, 300, (70, 33, 1)), 97
    print(f"\n[gpu layer head norm] embedding of {V} ids, {shape}", flush=True)
    inp, g = _group(shape, seed=6), torch.Generator().manual_seed(6)
    table = torch.randn(V, 256, generator=g).bfloat16().cuda()
    ids = [torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda() for n in (300, 70, 33, 1)]
    x = [torch.empty(len(t), 256, dtype=torch.bfloat16, device="cuda") for t in ids]
    for t, to in zip(ids, x):
        B.embed_fwd(t, table, to)
        assert torch.equal(to, table[t.long()])
    host = [t.float().cpu().numpy() for t in x]
    inp["x_p"], inp["x_s"] = host[0], host[1:]
    got, ref = DecoderLayer(inp).run_schedule(), _reference(inp)
    dtable = torch.zeros(V, 256, device="cuda")
    want, tol = np.zeros((V, 256)), np.zeros((V, 1))
    for t, dx, r in zip(ids, [got["dx_p"], *got["dx_s"]], [ref["dx_p"], *ref["dx_s"]]):
        ws = torch.empty(B.embed_bwd_workspace_size(len(t), V, 256), dtype=torch.uint8, device="cuda")
        B.embed_bwd(t, dx.bfloat16().contiguous(), dtable, ws=ws)
        at = t.cpu().numpy()
        np.add.at(want, at, r)
        # rounding dx to bf16, if it is not already, is 2^-8 of it more
        np.add.at(tol, at, np.full((len(at), 1), (TOL + 2.0 ** -8) * np.abs(r).max()))
    off = np.abs(dtable.double().cpu().numpy() - want) - tol
    assert off.max() <= 0, off.max()
