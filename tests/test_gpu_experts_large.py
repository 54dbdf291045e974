"""The experts' products in their largest tiles, 256 x 256 of eight waves: sizes
that the rules send there (checked on the CPU against the rules themselves), with
ends of 1 to 225 rows behind whole tiles, empty groups, widths off 64 and 256,
contractions from a part of a step to many steps, one and two pairs, gathered and
plain rows, written and added, and bad values next to good ones.  Bounds as in the
other tests of these products."""
import numpy as np
import pytest

from host_rules import answers, part
from test_gpu_experts import _check_all, _make, _say

# a tile's eight waves have 4 32-row blocks each, two waves' blocks in turn: an end
# of 1, 33, 65, .. rows leaves each of their counts to one of the waves
ENDS = [257, 289, 65, 97, 0, 385, 161, 705, 225, 256, 255, 0, 64, 32]
FEW = [1030, 511, 0, 1025, 290]
CASES = {  # sizes, in_width, out_width, rows to gather from, two pairs
    # forward products
    "fwd_pair": (ENDS, 136, 1544, 50, True), "fwd_pair_plain": (ENDS, 64, 1672, None, True),
    "fwd_part_of_a_step": (ENDS, 8, 1736, 90, True), "fwd_long": (FEW, 1032, 2056, 300, True),
    "fwd_one": (ENDS, 200, 2824, 70, False), "fwd_one_plain": (ENDS, 72, 2880, None, False),
    # rows' gradients
    "bwd_x_pair": (ENDS, 2824, 136, 50, True), "bwd_x_part_of_a_step": (ENDS, 3016, 8, None, True),
    "bwd_x_step": (ENDS, 2888, 64, 40, True), "bwd_x_long": (FEW, 5128, 1032, None, True),
    # weights' gradients
    "bwd_w_pair": (ENDS, 264, 776, 60, True), "bwd_w_plain": (ENDS, 520, 1288, None, True),
    "bwd_w_one": (ENDS, 520, 1096, 60, False), "bwd_w_one_plain": (ENDS, 776, 776, None, False)}
ALL = ([300, 257, 0, 705, 511, 640], 3208, 1544)  # every product of a pair


def _tiles(cases):
    """(rows, columns) of the tiles of fwd, bwd_x and bwd_w, by the library's rules."""
    code = """
typedef int hipError_t;
typedef int hipStream_t;
enum ExpertMode { kFwd = 0, kBwdX = 1, kBwdW = 2 };
struct ExpertArgs { int32_t E, rows, in_width, out_width, two; };
template <int MODE> int pairs(const ExpertArgs& a) { return a.two ? 2 : 1; }
template <int MODE, int BM, int BN, int MW, int NW, int STEP, int RING, bool TOKENS = false>
hipError_t launch_tiles(const ExpertArgs&, hipStream_t) {
  printf("%d %d ", BM, BN);
  return 0;
}
""" + part("kernels_experts.hip", "bool small_tiles(", "}  // namespace\n\nhipError_t launch_experts_fwd") + """
int main() {
  ExpertArgs a;
  int tokens;
  while (scanf("%d %d %d %d %d %d", &a.E, &a.rows, &a.in_width, &a.out_width, &a.two, &tokens) == 6) {
    launch_rows_of<kFwd>(a, a.out_width, pairs<kFwd>(a), 0);
    launch_rows_of<kBwdX>(a, a.in_width, 1, 0);
    if (tokens) launch_bwd_w<true>(a, 0); else launch_bwd_w<false>(a, 0);
    a.two = 0;  // as _check_all adds
    if (tokens) launch_bwd_w<true>(a, 0); else launch_bwd_w<false>(a, 0);
    printf("\\n");
  }
}
"""
    return answers(code, cases)


def _line(sizes, i, o, tokens, two):
    rows = sum(sizes) + (5 if tokens else 0)
    return len(sizes), rows, i, o, two, tokens is not None


def test_the_rules_pick_the_largest_tiles():
    got = dict(zip(CASES, _tiles([_line(*c) for c in CASES.values()])))
    at = {"fwd": slice(0, 2), "bwd_x": slice(2, 4), "bwd_w": slice(4, 6)}
    for name, tiles in got.items():
        way = next(w for w in at if name.startswith(w))
        assert tiles[at[way]] == [256, 256], (name, tiles)
    for tokens in (None, 400):
        assert _tiles([_line(*ALL, tokens, True)]) == [[256] * 8]
    # written and added, gathered and plain
    assert all(got[n][6:] == [256, 256] for n in ("bwd_w_plain", "bwd_w_one", "bwd_w_one_plain"))


def test_other_sizes_have_other_tiles():
    """The stubs do not answer the same for everything."""
    assert _tiles([(128, 8, 2048, 768, 1, 1)]) == [[32, 64, 32, 64, 128, 128, 128, 128]]
    assert _tiles([(8, 2000, 512, 512, 1, 1)])[0][:2] == [128, 128]


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_formulas(gpu, name):
    sizes, i, o, tokens, two = CASES[name]
    _say(f"large tiles, {name}: {i} x {o} tokens {tokens} two {two}")
    _check_all(_make(sizes, i, o, tokens=tokens, tail=5 if tokens else 0, seed=len(name)), i, o, two)


@pytest.mark.gpu
def test_a_bad_row_stays_in_its_group(gpu):
    """NaN and infinity in an expert's last row, in its weights and in the rows
    behind the last group; every contraction ends in a part of a step."""
    import torch
    from paper_2606_01143_amd import binding as B
    _say("large tiles, bad rows")
    (sizes, i, o), tail = ALL, 9
    s = _make(sizes, i, o, tail=tail, seed=3)
    at = np.concatenate([[0], np.cumsum(sizes)])
    last, rows = int(at[2]) - 1, int(at[-1]) + tail
    bad = {n: t.clone() for n, t in s.items() if n in ("x", "dy", "w")}
    bad["x"][last, i - 1], bad["dy"][last, o - 1] = float("inf"), float("nan")
    bad["x"][-tail:], bad["dy"][-tail:] = float("nan"), float("inf")
    bad["w"][3, i - 1, 0] = float("nan")
    out = []
    for t in (s, {**s, **bad}):
        y, y2 = (torch.zeros(rows, o, device="cuda").bfloat16() for _ in range(2))
        dx = torch.zeros(rows, i, device="cuda").bfloat16()
        dw, dw2 = (torch.zeros(6, i, o, device="cuda") for _ in range(2))
        B.experts_fwd(t["off"], t["x"], t["w"], y, w2=t["w2"], y2=y2)
        B.experts_bwd_x(t["off"], t["dy"], t["w"], dx, dy2=t["dy2"], w2=t["w2"])
        B.experts_bwd_w(t["off"], t["x"], t["dy"], dw, dy2=t["dy2"], dw2=dw2)
        torch.cuda.synchronize()
        out.append((y, y2, dx, dw, dw2))
    (y0, y20, dx0, dw0, dw20), (y, y2, dx, dw, dw2) = out
    third = slice(int(at[3]), int(at[4]))
    # the bad row's own products, and the bad weight's column, and nothing else
    assert not torch.isfinite(y[last]).any() and dx[last].isnan().all() and not torch.isfinite(y2[last]).any()
    assert y[third, 0].isnan().all() and dx[third, i - 1].isnan().all()
    for t, t0 in ((y, y0), (y2, y20), (dx, dx0)):
        t[last] = t0[last]
    y[third, 0], dx[third, i - 1] = y0[third, 0], dx0[third, i - 1]
    assert torch.equal(y, y0) and torch.equal(y2, y20) and torch.equal(dx, dx0)
    assert not torch.isfinite(dw[1, i - 1]).any() and dw[1, :, o - 1].isnan().all()
    assert not torch.isfinite(dw2[1, i - 1]).any()
    dw[1, i - 1], dw[1, :, o - 1], dw2[1, i - 1] = dw0[1, i - 1], dw0[1, :, o - 1], dw20[1, i - 1]
    assert torch.equal(dw, dw0) and torch.equal(dw2, dw20)


@pytest.mark.gpu
def test_repeats_and_graphs(gpu):
    """Bitwise the same in eager calls, on another stream and in four replays of a
    captured graph with eager work between."""
    import torch
    from paper_2606_01143_amd import binding as B
    _say("large tiles, graph")
    sizes, i, o = ALL
    s = _make(sizes, i, o, tokens=400, tail=5, seed=8)
    rows = sum(sizes) + 5
    bf = dict(dtype=torch.bfloat16, device="cuda")

    def outs():
        return [torch.zeros(rows, o, **bf), torch.zeros(rows, o, **bf), torch.zeros(rows, i, **bf),
                torch.zeros(6, i, o, device="cuda"), torch.zeros(6, i, o, device="cuda")]

    def call(r, stream=None):
        B.experts_fwd(s["off"], s["x"], s["w"], r[0], w2=s["w2"], y2=r[1], row_token=s["tok"], stream=stream)
        B.experts_bwd_x(s["off"], s["dy"], s["w"], r[2], dy2=s["dy2"], w2=s["w2"], stream=stream)
        B.experts_bwd_w(s["off"], s["x"], s["dy"], r[3], dy2=s["dy2"], dw2=r[4], row_token=s["tok"], overwrite=True,
                        stream=stream)
    want, other, held = outs(), outs(), outs()
    call(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(other, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(held)
    for _ in range(4):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held))
        call(other)
