"""Steps over the cache's other forms with every feature map and either sign of the scale at every head size, and the tile kernel over
packed rings of head size 128, which the plan takes from twice as many rows on; every test asserts which kernel ran."""
import numpy as np
import pytest
import torch

from oracle import rattn_oracle as orc
from paper_2506_15545_amd import binding as rb
from test_gpu_packed_rings import NAMES, check_out, oracle_step, step_inputs
from test_gpu_tree import CACHE, check, check_commit, make, np64, oracle, step
from test_gpu_tree_tiles import kernels, positions, some

pytestmark = pytest.mark.gpu
FORMS = [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)]


def ran(x, scale, tiles, **kw):
    assert kernels(lambda: step(x, scale, **kw)) == {"tree_tile_kernel" if tiles else "tree_kernel"}


@pytest.mark.parametrize("phi", ["relu", "identity"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,packed", FORMS)
def test_maps_direct(phi, D, dtype, packed):
    W = 21
    x = make(4, 30, 8, 2, D, W, dtype, [5, 21, 99, 20], packed, 9800, 1)      # chains longer than the window
    ran(x, 0.125, False, feature_map=phi)
    check(step(x, 0.125, feature_map=phi), oracle(x, W, 0.125, phi), dtype, x)
    keep = {n: x[n].clone() for n in CACHE if x[n] is not None}
    check_commit(x, keep, torch.tensor([29, 12, 3, -1], dtype=torch.int32, device="cuda"), W, phi)


@pytest.mark.parametrize("phi", ["relu", "identity"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("packed", [False, True])
def test_maps_tiles(phi, D, packed):
    N, W = 130, 21
    x = make(N, 64, 8, 2, D, W, "bf16", positions(N, W), packed, 9810, 2)
    ran(x, 0.125, True, feature_map=phi)
    ns = list(range(8))
    check(step(x, 0.125, feature_map=phi)[ns], oracle(some(x, ns), W, 0.125, phi), "bf16", x)


@pytest.mark.parametrize("scale", [-0.1, 2.0])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,packed", FORMS)
def test_scales_direct(scale, D, dtype, packed):
    W = 75
    x = make(4, 20, 8, 2, D, W, dtype, [10, 75, 200, 74], packed, 9820, 3)
    ran(x, scale, False)
    check(step(x, scale), oracle(x, W, scale), dtype, x)


@pytest.mark.parametrize("scale", [-0.1, 2.0])
@pytest.mark.parametrize("D", [64, 128])
def test_scales_tiles_over_packed_rings(scale, D):
    N, W = 260, 75
    x = make(N, 20, 8, 2, D, W, "bf16", positions(N, W), True, 9830, 3)
    ran(x, scale, True)
    ns = list(range(8))
    check(step(x, scale)[ns], oracle(some(x, ns), W, scale), "bf16", x)


@pytest.mark.parametrize("phi", ["softmax", "relu", "identity"])
@pytest.mark.parametrize("scale", [-0.1, 0.09])
@pytest.mark.parametrize("W,pos", [(40, [7, 40, 99]), (4097, [4096, 9000, 50])])    # a work-group for each ring, several
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_decode(phi, scale, W, pos, dtype):
    x, gains, _ = step_inputs(3, 6, 2, 128, W, dtype, pos, 9840)
    o_ref, _, _, S = oracle_step(x, gains, scale, W, phi)
    o = rb.rattn_decode_step_packed(*(x[n] for n in NAMES), *gains, softmax_scale=scale, feature_map=phi)
    check_out(o, o_ref, dtype, gains)
    assert float(np.abs(np64(x["state"]) - S).max()) <= 1e-5 * max(1.0, float(np.abs(S).max()))


@pytest.mark.parametrize("N,M,Hq,Hkv,W,spread", [
    (180, 33, 4, 1, 200, 1),             # 132 rows: a second work-group of one wave; chains
    (260, 17, 8, 2, 37, 3),              # 68 rows: the third wave has four of them
    (300, 64, 2, 1, 1, 2), (130, 64, 8, 2, 20, 1)])     # a window of one; chains longer than the window
def test_tiles_over_packed_rings_of_128(N, M, Hq, Hkv, W, spread):
    x = make(N, M, Hq, Hkv, 128, W, "bf16", positions(N, W), True, 9850 + M, spread)
    ran(x, 0.09, True)
    o = step(x, 0.09)
    assert torch.equal(o, step(x, 0.09))
    ns = [0, 1, 2, 3, 4, 5, 6, 7, N - 1]
    check(o[ns], oracle(some(x, ns), W, 0.09), "bf16", x)


def test_counts_over_packed_rings_of_128():
    N, M, W = 264, 19, 33
    pos = positions(N, W)
    pos[9], pos[17] = -1, -5
    x = make(N, M, 8, 2, 128, W, "bf16", pos, True, 9860, 3)
    count = [(M, 0, 4, -2, 17, 1, M + 5, 8)[i % 8] for i in range(N)]
    for name in ("q", "k", "v"):                 # what stands behind the last node is no number
        for n, c in enumerate(count):
            x[name][n, max(c, 0):] = float("nan")
    out, cnt = torch.full_like(x["q"], 7.0), torch.tensor(count, dtype=torch.int32, device="cuda")
    ran(x, 0.1, True, count=cnt)
    step(x, 0.1, count=cnt, out=out)
    live = [min(max(c, 0), M) if p >= 0 else 0 for c, p in zip(count, pos)]
    assert all(bool((out[n, c:] == 7.0).all()) for n, c in enumerate(live))
    ns = [2, 4, 5, 6, 7, 10, 12, N - 1]
    ref = oracle(some(x, ns), W, 0.1, count=[live[n] for n in ns])
    for i, n in enumerate(ns):
        if live[n]:
            check(out[n, :live[n]], ref[i, :live[n]], "bf16", x)


@pytest.mark.parametrize("D", [64, 128])
def test_captured_over_packed_rings(D):
    """A step of the tile kernel and the commit that follows it in one graph, replayed with eager work between the replays."""
    N, M, W = 260, 17, 100
    x = make(N, M, 8, 2, D, W, "bf16", positions(N, W), True, 9870, 2)
    last = torch.full((N,), M - 1, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([len(orc.tree_path(p, M - 1)) for p in x["parent"].cpu().numpy()], dtype=torch.int32, device="cuda")
    ran(x, 0.1, True)
    y = {n: (t.clone() if t is not None else None) for n, t in x.items()}

    def both(s, out):
        step(s, 0.1, out=out)
        rb.rattn_tree_commit(s["k"], s["v"], s["parent"], last, s["pos"], s["kr"], s["vr"], s["state"], k_scale=s["ks"], v_scale=s["vs"])

    out, want = torch.empty_like(x["q"]), torch.empty_like(x["q"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(x, out)
    for turn in range(4):
        out.fill_(float("nan"))
        graph.replay()
        both(y, want)
        assert torch.equal(out, want), turn
        for s in (x, y):
            s["pos"] += lengths
            s["q"].mul_(0.9)
        assert all(torch.equal(x[n].view(torch.uint8), y[n].view(torch.uint8)) for n in CACHE), turn
