"""The embedding's gradient in its longer spans, 32 and 64 sorted tokens a wave,
with one and several slabs of 512 columns, the last one partly used: runs inside a
span, runs that cross one border and runs over hundreds of spans, padding that ends
inside a span.  The span of each size is asked of the library's own rule on the CPU.
Bounds as in the other tests: each addition is off by at most 2^-24 of the sum of
magnitudes."""
import numpy as np
import pytest

from host_rules import answers, part
from test_gpu_embed import U32, _bwd, _dt, _ids, _say

# tokens, vocabulary, width, ids, type, span
CASES = [(17000, 900, 4096, "frequent", "bf16", 32), (19001, 128000, 3592, "frequent", "bf16", 32),
         (20011, 40, 3600, "any", "f32", 32), (26221, 3, 2568, "few", "bf16", 32), (19999, 700, 4088, "padded", "f32", 32),
         (33001, 900, 4096, "frequent", "f32", 64), (40003, 50000, 3592, "frequent", "bf16", 64),
         (37451, 7, 3600, "any", "bf16", 64), (33333, 11, 4088, "one", "f32", 64), (52500, 6000, 2568, "padded", "bf16", 64),
         (131073, 5000, 8, "frequent", "f32", 32), (300007, 9000, 8, "any", "bf16", 64), (140001, 5, 1032, "few", "f32", 64)]


def test_the_rule_picks_these_spans():
    code = part("kernels_embed.hip", "int embed_span(long n, long slabs) {", "// workspace: two buffers of keys") + """
int main() {
  long n, width;
  while (scanf("%ld %ld", &n, &width) == 2) printf("%d\\n", embed_span(n, (width / 8 + 63) / 64));
}
"""
    got = answers(code, [c[0::2][:2] for c in CASES])
    assert [g[0] for g in got] == [c[5] for c in CASES]


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,width,kind,dt,span", CASES)
def test_against_the_formulas(gpu, T, V, width, kind, dt, span):
    import torch
    _say(f"spans of {span}: T {T} V {V} width {width} {kind} {dt}")
    ids = _ids(kind, T, V, seed=T)
    valid = (ids >= 0) & (ids < V)
    g = torch.Generator(device="cuda").manual_seed(T + V)
    dy = torch.randn(T, width, generator=g, device="cuda").to(_dt(dt))
    before = torch.randn(V, width, generator=g, device="cuda")
    dev = torch.from_numpy(ids.astype(np.int64)).to(torch.int32).cuda()
    scale = float(np.float32(0.7))
    grads = [before.clone() for _ in range(2)]
    for t in grads:
        _bwd(dev, dy, t, scale)
    assert torch.equal(*grads)
    rows = torch.from_numpy(ids[valid]).cuda()
    count = torch.bincount(rows, minlength=V).double()
    keep = torch.from_numpy(valid).cuda()
    for c in range(0, width, 512):  # a slab at a time
        kept, was = dy[keep, c:c + 512].double(), before[:, c:c + 512].double()
        want = was.clone().index_add_(0, rows, kept * scale)
        mag = was.abs().index_add_(0, rows, kept.abs() * scale)
        off = (grads[0][:, c:c + 512].double() - want).abs() - (count[:, None] + 4) * U32 * mag
        assert (off <= 0).all(), f"columns {c} on: {off.max().item():.3e} over"
    untouched = count == 0
    assert torch.equal(grads[0][untouched], before[untouched])
