"""What a stack holds of its suffixes (schedule) and trajectories (dense) between
forward and backward: every layer's own saved activations and nothing that only
the next layer's input was for."""
import pytest
import torch

from synthetic.layer import LayerShape, make_stack_group

SHAPE = LayerShape(256, 4, 2, 64, 512, 40, (33, 70))


def _eight(rows, width):
    return rows * (width + -(-width // 32))


def _watch(monkeypatch, stack, seen):
    """Records, at a layer's backward, what every layer of the pass holds."""
    held = []  # the dicts of the forwards, in order
    for layer in stack.layers:
        forward, backward = layer._forward, layer._backward

        def _forward(x, pos0, attend, forward=forward, layer=layer):
            c = forward(x, pos0, attend)
            held.append((layer, c))
            return c

        def _backward(c, g, pos0, attend_bwd, dw, backward=backward):
            seen.append((pos0, g.shape[0], [(at, dict(d)) for at, d in held]))
            return backward(c, g, pos0, attend_bwd, dw)

        monkeypatch.setattr(layer, "_forward", _forward)
        monkeypatch.setattr(layer, "_backward", _backward)


def _no_output(seen):
    """No saved dict holds its layer's output: it is the next layer's input, which
    keeps what it needs of it, or the caller's."""
    assert seen
    for pos0, rows, held in seen:
        for _, c in held:
            assert "y" not in c, (pos0, rows, sorted(c))


def test_layers_hold_no_outputs(monkeypatch):
    """Both passes on the CPU, the layers' kernels replaced by stand-ins."""
    from paper_2606_01143_amd import binding as B
    from paper_2606_01143_amd.stack import DecoderStack
    monkeypatch.setattr(B, "gkv_cache_zero", lambda *a, **k: None)
    inp = make_stack_group(SHAPE, 3, seed=1)
    for saved in ("bf16", "int8"):
        stack = DecoderStack(inp, device="cpu", saved=saved)
        for layer in stack.layers:
            monkeypatch.setattr(layer, "_forward", lambda x, pos0, attend: {"y": x + 1, "q": x, "k": x, "v": x})
            monkeypatch.setattr(layer, "_backward", lambda c, g, pos0, attend_bwd, dw: g + 1)
            monkeypatch.setattr(layer, "_dims_for", lambda n: (None, None, (None, None)))
        seen = []
        _watch(monkeypatch, stack, seen)
        for run in (stack.run_schedule, stack.run_dense):
            out = run()
            # the outputs reach the caller all the same
            for y, x in zip(out["y_s"], stack.x_s):
                assert torch.equal(y, x + 1 + 1 + 1)
            assert torch.equal(out["y_p"], stack.x_p + 1 + 1 + 1)
        _no_output(seen)


@pytest.mark.gpu
@pytest.mark.parametrize("saved", ["bf16", "int8"])
def test_bytes_of_a_suffix(gpu, monkeypatch, saved):
    """A suffix's saved tensors are those of the layer's form, to the byte."""
    from paper_2606_01143_amd.stack import DecoderStack
    print(f"\n[gpu stack saved] {saved}", flush=True)
    stack = DecoderStack(make_stack_group(SHAPE, 3, seed=2), saved=saved)
    seen = []
    _watch(monkeypatch, stack, seen)
    stack.run_schedule()
    stack.run_dense()
    torch.cuda.synchronize()
    _no_output(seen)
    hid, mid, hq, hkv, d = SHAPE.hidden, SHAPE.intermediate, SHAPE.num_q_heads, SHAPE.num_kv_heads, SHAPE.head_dim
    for pos0, _, held in seen:
        for layer, c in held:
            rows = c["q"].shape[0]
            own = rows * (2 * 2 * hq * d + 2 * 2 * hkv * d + 4 * (hq + 2))  # q, o, k, v, LSE, the norms' statistics
            if saved == "int8":
                own += 2 * _eight(rows, hid) + 2 * _eight(rows, mid)  # x, h, g, u
            else:
                own += rows * 2 * (4 * hid + 3 * mid)  # x, n1, h, n2, g, u, m
            assert sum(t.numel() * t.element_size() for t in c.values()) == own, (pos0, sorted(c))
