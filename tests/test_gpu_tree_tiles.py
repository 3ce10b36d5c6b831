"""Tree steps of many rows in many pairs (sequence, KV head), whose keys come through LDS: some of their sequences against the fp64
oracle, all of them against steps of a few sequences, which fetch their keys themselves."""
import numpy as np
import pytest
import torch

from test_gpu_tree import CACHE, check, make, np64, oracle, step

pytestmark = pytest.mark.gpu
PER = ("q", "k", "v", "parent", "pos", "kr", "vr", "ks", "vs", "state")


def some(x, ns):
    return {n: t[ns].contiguous() if n in PER and t is not None else t for n, t in x.items()}


def kernels(f):
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA]) as prof:
        f()
        torch.cuda.synchronize()
    return {name for e in prof.events() for name in ("tree_tile_kernel", "tree_kernel") if name in e.name}


def positions(N, W):
    """Empty, filling, just full and wrapped windows, and long sequences, in turn."""
    return [(0, W // 2, max(W - 3, 0), W, W + 1, 2 * W + 7, 40 * W + 5, 5)[i % 8] for i in range(N)]


SHAPES = [  # N, M, Hq, Hkv, W, spread: pairs * ceil(M G / 64) above 512
    (65, 17, 16, 4, 37, 3),              # 68 rows: the third wave has four of them
    (33, 13, 40, 8, 130, 2),             # 65 rows
    (130, 33, 4, 1, 200, 1),             # 132 rows: a second work-group of one wave; chains
    (130, 64, 4, 2, 20, 1),              # chains longer than the window
    (27, 64, 20, 1, 96, 5),              # 20 query heads of a KV head: gains from memory
    (520, 64, 2, 1, 1, 2),               # a window of one
    (65, 24, 32, 8, 64, 4),              # 96 rows, a window of one tile
    (40, 33, 40, 8, 130, 3), (64, 33, 32, 8, 50, 1)]   # more work-groups than run at once, of 64 sequences at most: the longest first


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,M,Hq,Hkv,W,spread", SHAPES)
def test_step(N, M, Hq, Hkv, D, W, spread, packed):
    print(f"N={N} M={M} Hq={Hq} Hkv={Hkv} D={D} W={W} packed={packed}", flush=True)
    x = make(N, M, Hq, Hkv, D, W, "bf16", positions(N, W), packed, 9000 + M + W, spread)
    scale = D ** -0.5
    keep = {n: x[n].clone() for n in CACHE if x[n] is not None}
    o = step(x, scale)
    for n, t in keep.items():
        assert torch.equal(t.view(torch.uint8), x[n].view(torch.uint8)), n
    assert torch.equal(o, step(x, scale))
    ns = [0, 1, 2, 3, 4, 5, 6, N - 1] if M * Hq * Hkv < 400 else [0, 2, 4, N - 1]
    check(o[ns], oracle(some(x, ns), W, scale), "bf16", x)
    few = torch.cat([step(some(x, slice(i, i + 8)), scale) for i in range(0, N, 8)])
    top = max(1.0, float(x["gs"].abs().max()), float(x["gr"].abs().max()))
    assert float((o.float() - few.float()).abs().max()) <= 2 * 2e-2 * top     # either is within 2e-2 of the formula


def test_which_calls_take_it():
    """More than 256 work-groups of 64 rows (512 with packed rings of head size 128), bf16, more than 64 rows."""
    for N, M, Hq, D, dtype, packed, tiles in ((129, 17, 4, 128, "bf16", False, True), (128, 17, 4, 128, "bf16", False, False),
                                              (400, 16, 4, 128, "bf16", False, False), (129, 17, 4, 128, "f32", False, False),
                                              (129, 17, 4, 128, "bf16", True, False), (257, 17, 4, 128, "bf16", True, True),
                                              (129, 17, 4, 64, "bf16", True, True)):
        x = make(N, M, Hq, 1, D, 8, dtype, [50] * N, packed, 9100)
        step(x, 0.1)
        assert kernels(lambda: step(x, 0.1)) == {"tree_tile_kernel" if tiles else "tree_kernel"}, (N, M, D, dtype, packed)


@pytest.mark.parametrize("phi", ["relu", "identity"])
@pytest.mark.parametrize("packed", [False, True])
def test_feature_maps(phi, packed):
    N, W = 130, 21
    x = make(N, 64, 8, 2, 64, W, "bf16", positions(N, W), packed, 9200, 2)
    ns = list(range(8))
    check(step(x, 0.125, feature_map=phi)[ns], oracle(some(x, ns), W, 0.125, phi), "bf16", x)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [-0.1, 2.0])
def test_scales(D, scale):
    N, W = 130, 75
    x = make(N, 20, 8, 2, D, W, "bf16", positions(N, W), False, 9300, 3)
    ns = list(range(8))
    check(step(x, scale)[ns], oracle(some(x, ns), W, scale), "bf16", x)


def test_without_gains_and_gains_of_any_alignment():
    N, W, D = 130, 40, 128
    x = make(N, 18, 8, 2, D, W, "bf16", positions(N, W), False, 9400, 3)
    ns, ones = list(range(8)), torch.ones(8, D, device="cuda")
    check(step({**x, "gs": None, "gr": None}, 0.1)[ns], oracle(some({**x, "gs": ones, "gr": ones}, ns), W, 0.1), "bf16", {**x, "gs": ones, "gr": ones})
    ref = step(x, 0.1)
    odd = {}
    for n in ("gs", "gr"):
        flat = torch.empty(8 * D + 1, device="cuda")
        odd[n] = flat[1:].view(8, D)
        odd[n].copy_(x[n])
    assert torch.equal(step({**x, **odd}, 0.1), ref)


@pytest.mark.parametrize("N,M,Hkv", [(132, 19, 2), (48, 40, 8)])
def test_counts_and_sequences_without_work(N, M, Hkv):
    W = 33
    pos = positions(N, W)
    pos[9], pos[17] = -1, -5
    x = make(N, M, 4 * Hkv, Hkv, 128, W, "bf16", pos, False, 9500, 3)
    count = [(M, 0, 4, -2, 17, 1, M + 5, 8)[i % 8] for i in range(N)]
    for name in ("q", "k", "v"):                 # what stands behind the last node is no number
        for n, c in enumerate(count):
            x[name][n, max(c, 0):] = float("nan")
    out = torch.full_like(x["q"], 7.0)
    step(x, 0.1, count=torch.tensor(count, dtype=torch.int32, device="cuda"), out=out)
    live = [min(max(c, 0), M) if p >= 0 else 0 for c, p in zip(count, pos)]
    assert all(bool((out[n, c:] == 7.0).all()) for n, c in enumerate(live))
    ns = [n for n in (2, 4, 5, 6, 7, 10, 12, N - 1)]
    ref = oracle(some(x, ns), W, 0.1, count=[live[n] for n in ns])
    for i, n in enumerate(ns):
        if live[n]:
            check(out[n, :live[n]], ref[i, :live[n]], "bf16", x)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan"), 3.0e38])
def test_other_branches_and_left_keys_do_not_matter(bad, packed):
    N, M, W = 66, 33, 70
    x = make(N, M, 16, 8, 64, W, "bf16", [100, 17] * (N // 2), packed, 9600, 1)
    x["parent"][:, :8] = torch.tensor([-1, 0, 0, 2, 3, -1, 5, 6], dtype=torch.int32, device="cuda")
    x["parent"][:, 8:] = 7
    clean = step(x, 0.125)
    x["k"][:, 1, :, 5], x["v"][:, 1, :, 7] = bad, bad            # node 1: seen by itself alone
    x["v"][0, 5] = bad                                           # nodes 5 to 32 of the first sequence
    if not packed:
        x["kr"][1, :, 25, 3], x["vr"][1, :, 20:29] = bad, bad    # slots behind the 17 tokens
    o = step(x, 0.125)
    # Rows that the kernel forms again, key by key, differ from the tiles' by what either differs from the formula (2e-2 for both, as
    # above), and then either is rounded: by 2^-8 of its value, so that two roundings are one step, 2^-5 from |o| = 4 on
    close = lambda a, b: bool(((a.float() - b.float()).abs() <= 2e-2 + 2 * 2.0 ** -8 * b.float().abs()).all())
    rest = [0, 2, 3, 4]
    assert close(o[:, rest], clean[:, rest]) and close(o[1:, 5:], clean[1:, 5:])
    ns = [0, 1]
    with np.errstate(all="ignore"):
        ref = oracle(some(x, ns), W, 0.125)
    got = np64(o[ns])
    if not np.isfinite(bad):
        assert np.array_equal(np.isfinite(got), np.isfinite(ref))
    fin = np.isfinite(ref) & np.isfinite(got)
    if np.isfinite(bad):     # rows that see it: (3e38 P)^2, a term of the norm's fp32 sum, passes 3.4e38 unless P < 6.2e-20, and 1 / inf = 0
        fin[:, 1] = fin[0, 5:] = False
    assert float(np.abs(np.where(fin, got - ref, 0.0)).max()) <= 4e-2


def test_captured():
    N, M, W = 130, 17, 100
    x = make(N, M, 16, 4, 128, W, "bf16", positions(N, W), False, 9700, 2)
    out = torch.empty_like(x["q"])
    step(x, 0.1, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(x, 0.1, out=out)
    for turn in range(3):
        x["pos"] += 1
        x["q"].mul_(0.9)
        out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(out, step(x, 0.1)), turn


def test_calls_stay_inside_their_buffer():
    N, M, W, G = 130, 17, 100, 4096
    x = make(N, M, 16, 4, 128, W, "bf16", positions(N, W), False, 9800, 2)
    n = x["q"].numel() * 2
    full = torch.full((2 * G + n,), 0xA5, dtype=torch.uint8, device="cuda")
    ref = step(x, 0.1)
    assert torch.equal(step(x, 0.1, out=full[G:G + n].view(torch.bfloat16).view(x["q"].shape)), ref)
    assert bool((full[:G] == 0xA5).all()) and bool((full[G + n:] == 0xA5).all())
