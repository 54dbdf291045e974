"""Sizes past 32 bits (CPU): the C calls take int32, of which ctypes would pass
the low bits, so that a call would do the first few rows and say nothing."""
import pytest
import torch

from paper_2606_01143_amd import binding as B

FAR = (1 << 32) + 5


def _t(*shape, dt=torch.bfloat16):
    return torch.empty(*shape, dtype=dt, device="meta")  # no memory behind it


def _i(*shape):
    return _t(*shape, dt=torch.int32)


OFF = _i(5)
CALLS = {
    "heads fwd": lambda: B.head_norm_rope_fwd(_t(FAR, 1, 2), _t(FAR, 1, 2), _t(2), _t(2), _t(FAR, 1, 2),
                                              _t(FAR, 1, 2), 0, 1e4),
    "heads fwd position": lambda: B.head_norm_rope_fwd(_t(3, 1, 2), _t(3, 1, 2), _t(2), _t(2), _t(3, 1, 2),
                                                       _t(3, 1, 2), FAR, 1e4),
    "heads bwd": lambda: B.head_norm_rope_bwd(*(_t(FAR, 1, 2) for _ in range(2)), _t(2), _t(2),
                                              *(_t(FAR, 1, 2) for _ in range(4)), _t(2, dt=torch.float32),
                                              _t(2, dt=torch.float32), 0, 1e4),
    "embed fwd": lambda: B.embed_fwd(_i(FAR), _t(9, 8), _t(FAR, 8)),
    "embed fwd vocabulary": lambda: B.embed_fwd(_i(3), _t(FAR, 8), _t(3, 8)),
    "embed bwd": lambda: B.embed_bwd(_i(FAR), _t(FAR, 8), _t(9, 8, dt=torch.float32)),
    "plan": lambda: B.experts_plan(4, _i(FAR, 1), OFF, _i(FAR), _i(FAR, 1)),
    "experts fwd": lambda: B.experts_fwd(OFF, _t(9, 8), _t(4, 8, 8), _t(FAR, 8), row_token=_i(FAR)),
    "experts fwd source": lambda: B.experts_fwd(OFF, _t(FAR, 8), _t(4, 8, 8), _t(9, 8), row_token=_i(9)),
    "experts bwd x": lambda: B.experts_bwd_x(OFF, _t(FAR, 8), _t(4, 8, 8), _t(FAR, 8)),
    "experts bwd w": lambda: B.experts_bwd_w(OFF, _t(FAR, 8), _t(FAR, 8), _t(4, 8, 8, dt=torch.float32)),
    "combine fwd": lambda: B.experts_combine_fwd(_t(FAR, 8), _i(3, 2), None, _t(3, 8)),
    "combine bwd": lambda: B.experts_combine_bwd(_t(3, 8), None, _i(3, 2), None, _t(FAR, 8), None),
    "heads workspace": lambda: B.head_norm_rope_bwd_workspace_size(FAR, 1, 1, 64),
    "embed workspace": lambda: B.embed_bwd_workspace_size(FAR, 9, 8),
    "plan workspace": lambda: B.experts_plan_workspace_size(4, 1, FAR)}


@pytest.mark.parametrize("name", list(CALLS))
def test_a_size_past_32_bits(name):
    with pytest.raises(ValueError, match=f"a size of {FAR}"):
        CALLS[name]()
