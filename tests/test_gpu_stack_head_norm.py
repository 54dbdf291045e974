"""A stack whose layers normalise their queries and keys per head, through the
schedule (with and without offload) and dense, against the same stack in 64 bits
with gradients by autograd; the gate is the other stacks' (max-abs-relative 2e-2
in bf16).  One stack has such layers only, the other every second."""
import numpy as np
import pytest
import torch

from oracle.compare import max_abs_rel
from oracle.layer import _tail, attention, rms, rope
from synthetic.layer import LayerShape, make_stack_group

TOL = 2e-2
SHAPE = LayerShape(256, 4, 2, 64, 512, 200, (70, 33, 1))


def _group(shape, normed, seed):
    """A stack of len(normed) layers, with gains where the entry is true."""
    inp = make_stack_group(shape, len(normed), seed=seed)
    rng = np.random.default_rng(seed)
    for l, has in enumerate(normed):
        gains = {k: torch.from_numpy(1 + 0.3 * rng.standard_normal(shape.head_dim)).bfloat16().float().numpy()
                 for k in ("gq", "gk")}
        if has:
            inp["weights"][l] = dict(inp["weights"][l], **gains)
    return inp


def _reference(inp):
    shp = inp["shape"]
    t64 = lambda x, grad=False: torch.tensor(np.asarray(x, dtype=np.float64), requires_grad=grad)
    Ws = [{k: t64(v, True) for k, v in w.items()} for w in inp["weights"]]
    P, hq, hkv, d = shp.prefix_len, shp.num_q_heads, shp.num_kv_heads, shp.head_dim
    y_s, dx_s, dx_p, y_p = [], [], 0, None
    for x_s, dy_s, dy_p in zip(inp["x_s"], inp["dy_s"], inp["dy_p"]):
        x0 = x = t64(np.concatenate([inp["x_p"], x_s]), True)
        L = x.shape[0]
        pos, visible = torch.arange(L), torch.tril(torch.ones(L, L, dtype=torch.bool))
        for W in Ws:
            n = rms(x, shp.norm_eps)

            def head(w, g, h):
                v = (n @ W[w]).view(L, h, d)
                return rope(rms(v, shp.norm_eps) * W[g] if g in W else v, pos, shp.rope_theta)
            x = _tail(x, attention(head("wq", "gq", hq), head("wk", "gk", hkv), (n @ W["wv"]).view(L, hkv, d), visible),
                      W, shp)
        x.backward(t64(np.concatenate([dy_p, dy_s])))
        dx_p = dx_p + x0.grad[:P].numpy()
        dx_s.append(x0.grad[P:].numpy())
        y_s.append(x[P:].detach().numpy())
        y_p = x[:P].detach().numpy()
    return {"y_p": y_p, "y_s": y_s, "dx_p": dx_p, "dx_s": dx_s,
            "dw": [{k: v.grad.numpy() for k, v in W.items()} for W in Ws]}


def _np(t):
    return t.float().cpu().numpy().astype(np.float64)


def _check(got, ref, what):
    errs = {"y_p": max_abs_rel(_np(got["y_p"]), ref["y_p"]), "dx_p": max_abs_rel(_np(got["dx_p"]), ref["dx_p"])}
    for i, (y, dx) in enumerate(zip(got["y_s"], got["dx_s"])):
        errs[f"y_s{i}"] = max_abs_rel(_np(y), ref["y_s"][i])
        errs[f"dx_s{i}"] = max_abs_rel(_np(dx), ref["dx_s"][i])
    for l, (dw, rw) in enumerate(zip(got["dw"], ref["dw"])):
        assert set(dw) == set(rw), f"{what}: layer {l} has {sorted(dw)}"
        errs.update({f"L{l}.d{k}": max_abs_rel(_np(v), rw[k]) for k, v in dw.items()})
    assert not {k: v for k, v in errs.items() if not v <= TOL}, f"{what}: {errs}"


@pytest.mark.gpu
@pytest.mark.parametrize("normed", [(True, True, True), (True, False, True)], ids=["all", "mixed"])
def test_schedule_offload_and_dense(gpu, normed):
    from paper_2606_01143_amd.stack import DecoderStack, HbmBudget
    print(f"\n[gpu stack head norm] {normed} {SHAPE}", flush=True)
    inp = _group(SHAPE, normed, seed=21)
    ref = _reference(inp)
    plain = DecoderStack(inp).run_schedule()
    _check(plain, ref, "schedule")
    _check(DecoderStack(inp).run_dense(), ref, "dense")
    flat = lambda o: [o["y_p"], o["dx_p"], *o["y_s"], *o["dx_s"], *(w for dw in o["dw"] for w in dw.values())]
    for budget in (None, HbmBudget(limit=0)):
        st = DecoderStack(inp, offload=True, budget=budget)
        for _ in range(2):
            out = st.run_schedule()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(flat(plain), flat(out)))
        assert st.stats["pool_fallbacks"] == 0
        packed = [sum(h.numel() * h.element_size() for h in host.values()) for host in st._host]
        assert packed == st.dormant_bytes_of


def test_gains_are_kept_and_counted():
    from paper_2606_01143_amd.stack import DecoderStack
    st = DecoderStack(_group(SHAPE, (True, False), seed=1), device="cpu")
    assert [layer.head_norm for layer in st.layers] == [True, False]
    assert set(st.layers[0].w) - set(st.layers[1].w) == {"gq", "gk"}
    # 200 rows of 4 query and 2 key heads of 64 in bf16, before their norm
    assert st.dormant_bytes_of[0] - st.dormant_bytes_of[1] == 200 * 6 * 64 * 2
    assert st.layer_dormant_bytes == st.dormant_bytes_of[0] and st.dormant_bytes == sum(st.dormant_bytes_of)
    assert st.layers[0].ws_heads is st.ws_heads


def test_gains_go_together():
    from paper_2606_01143_amd.stack import DecoderStack
    inp = _group(SHAPE, (True, True), seed=1)
    del inp["weights"][1]["gk"]
    with pytest.raises(ValueError, match="go together"):
        DecoderStack(inp, device="cpu")
