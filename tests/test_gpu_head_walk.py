"""The per-head norm's row kernels where a wave has more to do than one round of
heads: several rounds of a token (its angles kept, the next rows loaded ahead,
from queries to keys), and several tokens (angles formed again, gain gradients
kept over all of them).  Which sizes do that is asked of the library's own rules
on the CPU.  Tolerances as in the other tests of these kernels: a gain gradient's
sum is at most 64 terms deep here (rounds of a wave, waves of a workgroup, twelve
partials and six joins)."""
import numpy as np
import pytest

from host_rules import answers, part
from test_gpu_head_norm_rope import _check, _dt, _inputs, _run, _say

# tokens, query and key heads, head dim: two and more tokens a wave, of two to five
# rounds of heads each; shares of two to four rounds; lanes without a value
CASES = [(5000, 32, 4, 128, "bf16"), (4200, 20, 5, 96, "bf16"), (4200, 8, 8, 256, "bf16"), (8300, 16, 8, 64, "bf16"),
         (4200, 32, 4, 128, "f32"), (4200, 8, 8, 256, "f32"), (5000, 3, 1, 80, "f32"), (9000, 1, 1, 16, "bf16"),
         (1500, 32, 8, 128, "bf16"), (1300, 33, 9, 128, "f32"), (700, 40, 40, 256, "f32")]
SHARES = [(1500, 32, 8, 128, "bf16"), (1300, 33, 9, 128, "f32"), (700, 40, 40, 256, "f32")]  # of a token's heads


def _walk(tokens, hq, hkv, d):
    """Rounds of a token, shares it is cut into, and rounds of a share."""
    code = """
struct HeadArgs { int32_t tokens, hq, hkv, d; };
""" + part("kernels_heads.hip", "int row_lanes(int d) {", "// the instantiation for the head dim's lanes per row") + """
int main() {
  HeadArgs a;
  while (scanf("%d %d %d %d", &a.tokens, &a.hq, &a.hkv, &a.d) == 4) {
    const int heads = 64 / row_lanes(a.d), rounds = (a.hq + heads - 1) / heads + (a.hkv + heads - 1) / heads;
    const int parts = head_parts(a);
    printf("%d %d %d\\n", rounds, parts, (rounds + parts - 1) / parts);
  }
}
"""
    return answers(code, [(tokens, hq, hkv, d)])[0]


@pytest.mark.parametrize("T,hq,hkv,d,dt", CASES)
def test_the_sizes_walk(T, hq, hkv, d, dt):
    rounds, parts, per = _walk(T, hq, hkv, d)
    # the forward has at most 4096 waves, the backward as many as 3 (fp32: 2) workgroups on 256 CUs
    assert per > 1
    assert T * parts > 4 * 256 * (3 if dt == "bf16" else 2) or (T, hq, hkv, d, dt) in SHARES
    if (T, hq, hkv, d, dt) in SHARES:
        assert 1 < parts < rounds
    else:
        assert parts == 1 and T > 4096


@pytest.mark.gpu
@pytest.mark.parametrize("T,hq,hkv,d,dt", CASES)
def test_against_the_formulas(gpu, T, hq, hkv, d, dt):
    import torch
    _say(f"walk, T {T} heads {hq}/{hkv} d {d} {dt}")
    # packed suffixes: positions that start again, so that a wave's tokens have angles of their own
    pos = (np.arange(T) * 7 + 3) % 2531
    i = _inputs(T, hq, hkv, d, _dt(dt), seed=T + d, positions=pos)
    got = _run(i, 4099, 1e-6)
    _check(i, got, pos + 4099.0, 1e-6)
    rest = got["grad"][:, (hq + hkv) * d:]
    assert torch.equal(rest, torch.full_like(rest, 7.0))
    again = _run(i, 4099, 1e-6)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.gpu
def test_a_bad_row_stays_in_its_row(gpu):
    """A NaN in a row that a wave holds between others, before and behind it."""
    import torch
    T, hq, hkv, d = 5000, 20, 5, 128
    _say(f"walk, bad rows, T {T}")
    i = _inputs(T, hq, hkv, d, torch.bfloat16, seed=9)
    clean = _run(i, 0, 1e-6)
    i["x"][17, 9 * d + 5] = float("nan")               # q head 9, a token whose wave has another behind it
    i["x"][4700, (hq + 4) * d + 1] = float("inf")      # k head 4, a wave's second token
    got = _run(i, 0, 1e-6)
    for n, t, h in (("q", 17, 9), ("k", 4700, 4)):
        for w in ("y", "d"):
            a, b = got[w + n].clone(), clean[w + n].clone()
            assert not torch.isfinite(a[t, h]).all()
            a[t, h] = b[t, h] = 0
            assert torch.equal(a, b), w + n
