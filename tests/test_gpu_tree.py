"""Trees of drafted tokens: the step over rings and state that it only reads, and the accepted path's entry into them, against the
fp64 oracle and against the calls that the cache's other users make."""
import ctypes
import math

import numpy as np
import pytest
import torch

import parity_metrics as pm

from oracle import rattn_oracle as orc
from paper_2506_15545_amd import binding as rb, synth

pytestmark = pytest.mark.gpu
np64 = lambda t: t.detach().cpu().to(torch.float64).numpy()
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CACHE = ("kr", "vr", "ks", "vs", "state")


def make(N, M, Hq, Hkv, D, W, dtype, pos, packed, seed, spread=3):
    """Inputs of a step: parents among the `spread` nodes before each, rings (packed or not) and state for positions pos."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, dt=DT[dtype]: torch.randn(*s, generator=g).to(dt).cuda()
    x = dict(q=r(N, M, Hq, D), k=r(N, M, Hkv, D), v=r(N, M, Hkv, D))
    back = torch.randint(0, spread, (N, M), generator=g)
    x["parent"] = torch.clamp(torch.arange(M) - 1 - back, min=-1).to(torch.int32).contiguous().cuda()
    x["pos"] = torch.tensor(pos, dtype=torch.int32, device="cuda")
    x["kr"], x["vr"], x["ks"], x["vs"] = r(N, Hkv, W, D), r(N, Hkv, W, D), None, None
    if packed:
        x["kr"], x["ks"], x["vr"], x["vs"] = rb.rattn_ring_pack(x["kr"], x["vr"])
    std = torch.sqrt(torch.clamp(x["pos"].float() - W, min=0.0) * math.e) / D
    x["state"] = r(N, Hkv, D, D, dt=torch.float32) * std.view(N, 1, 1, 1)
    x["gs"], x["gr"] = (1.0 + 0.25 * r(Hq, D, dt=torch.float32) for _ in range(2))
    return x


def ring_values(x):
    if x["ks"] is None:
        return np64(x["kr"]), np64(x["vr"])
    return orc.packed_values(np64(x["kr"]), np64(x["ks"])), orc.packed_values(np64(x["vr"]), np64(x["vs"]))


def step(x, scale, **kw):
    return rb.rattn_tree_step(x["q"], x["k"], x["v"], x["parent"], x["pos"], x["kr"], x["vr"], x["state"], x["gs"], x["gr"],
                              softmax_scale=scale, k_scale=x["ks"], v_scale=x["vs"], **kw)


def oracle(x, W, scale, phi="softmax", count=None):
    kr, vr = ring_values(x)
    return orc.tree_step(np64(x["q"]), np64(x["k"]), np64(x["v"]), x["parent"].cpu().numpy(), x["pos"].tolist(), kr, vr, np64(x["state"]), W,
                         scale=scale, gamma_swa=np64(x["gs"]), gamma_rla=np64(x["gr"]), feature_map=phi, count=count)


def check(o, ref, dtype, x, what="o"):
    top = max(1.0, float(x["gs"].abs().max()), float(x["gr"].abs().max()))
    if dtype == "bf16":
        pm.assert_out_bf16(np64(o), ref, gain_scale=top, what=what)
    else:   # the layer's bar for fp32 outputs of unit scale
        err = float(np.abs(np64(o) - ref).max())
        print(f"{what}: max-abs {err:.2e}", flush=True)
        assert err <= 1e-4 * top


SHAPES = [  # N, M, Hq, Hkv, W, pos, spread
    (1, 1, 1, 1, 1, [0], 1), (2, 1, 4, 2, 5, [0, 9], 1), (3, 5, 2, 2, 1, [0, 1, 7], 2), (3, 9, 3, 1, 4, [0, 3, 40], 1),
    (4, 7, 4, 2, 37, [0, 33, 37, 200], 3),               # windows that fill, and wrap, inside the tree
    (2, 33, 2, 1, 20, [10, 77], 1),                      # chains longer than the window
    (2, 64, 1, 1, 64, [63, 64], 1), (2, 64, 1, 1, 63, [64, 500], 1), (1, 64, 6, 1, 100, [99], 9),
    (2, 17, 20, 1, 130, [5, 1000], 4), (3, 13, 5, 1, 65, [64, 65, 66], 2),   # rows that no tile of 16 divides
    (9, 3, 8, 8, 96, [40 * i for i in range(9)], 2),     # 72 pairs: no multiple of the XCDs
    (1, 6, 4, 1, 2049, [5000], 2), (2, 40, 8, 2, 700, [300, 9999], 6),       # several work-groups for a ring
    (1, 5, 2, 1, 4321, [9000], 1), (2, 8, 4, 1, 4096, [4095, 4097], 2), (1, 30, 4, 2, 4100, [70000], 3),
    (3, 4, 4, 1, 200, [0, 199, 999], 2), (2, 8, 8, 2, 300, [299, 5000], 2),  # four waves: short windows, many pairs
    (70, 3, 16, 4, 64, [7 * i for i in range(70)], 1), (65, 7, 16, 4, 333, [31 * i for i in range(65)], 3)]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("N,M,Hq,Hkv,W,pos,spread", SHAPES)
def test_step(N, M, Hq, Hkv, D, W, dtype, pos, spread, packed):
    print(f"N={N} M={M} Hq={Hq} Hkv={Hkv} D={D} W={W} {dtype} packed={packed}", flush=True)
    x = make(N, M, Hq, Hkv, D, W, dtype, pos, packed, 7000 + M + W, spread)
    scale = D ** -0.5
    keep = {n: x[n].clone() for n in CACHE if x[n] is not None}
    o = step(x, scale)
    check(o, oracle(x, W, scale), dtype, x)
    for n, t in keep.items():     # the cache is only read
        assert torch.equal(t.view(torch.uint8), x[n].view(torch.uint8)), n
    assert torch.equal(o, step(x, scale))


@pytest.mark.parametrize("phi", ["relu", "identity"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
def test_feature_maps(phi, dtype, packed):
    W = 21
    x = make(3, 30, 4, 2, 64, W, dtype, [5, 21, 99], packed, 7100, 2)
    check(step(x, 0.125, feature_map=phi), oracle(x, W, 0.125, phi), dtype, x)
    keep = {n: x[n].clone() for n in CACHE if x[n] is not None}
    accepted = torch.tensor([29, 12, 3], dtype=torch.int32, device="cuda")
    check_commit(x, keep, accepted, W, phi)


def check_commit(x, keep, accepted, W, phi="softmax"):
    """x's cache after a commit against the oracle's, from `keep`; rings to the bit.  State: sums of up to 64 fp32 multiply-adds of
    terms no larger than the state's entries."""
    y = {**x, **keep}
    kr, vr = ring_values(y)
    wk, wv, wS = orc.tree_commit(np64(x["k"]), np64(x["v"]), x["parent"].cpu().numpy(), accepted.tolist(), x["pos"].tolist(), kr, vr,
                                 np64(y["state"]), W, phi)
    rb.rattn_tree_commit(x["k"], x["v"], x["parent"], accepted, x["pos"], x["kr"], x["vr"], x["state"], k_scale=x["ks"], v_scale=x["vs"],
                         feature_map=phi)
    if x["ks"] is None:
        assert np.array_equal(np64(x["kr"]), wk) and np.array_equal(np64(x["vr"]), wv)
    else:
        for c, s, want, old, new in (("kr", "ks", wk, kr, "k"), ("vr", "vs", wv, vr, "v")):
            got = orc.packed_values(np64(x[c]), np64(x[s]))
            rows = np.any(want != old, -1)            # slots that a token took
            assert np.array_equal(got[~rows], old[~rows])
            assert np.array_equal(got[rows], orc.packed_values(*orc.pack_rows(want[rows])))
    err = float(np.abs(np64(x["state"]) - wS).max())
    assert err <= 1e-5 * max(1.0, float(np.abs(wS).max())), err


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("N,M,Hkv,W,pos,spread,accepted", [
    (1, 1, 1, 1, [0], 1, [0]), (3, 1, 2, 6, [5, 6, 7], 1, [0, -1, 0]), (4, 12, 2, 9, [0, 3, 9, 77], 1, [11, 5, 11, 0]),
    (2, 64, 1, 10, [4, 100], 1, [63, 63]),               # most of the path leaves at once
    (5, 20, 3, 50, [0, 45, 50, 51, 3000], 3, [19, 17, -1, 19, 64]),    # (one that is no node)
    (9, 6, 8, 130, [31 * i for i in range(9)], 2, [5, 4, 3, 2, 1, 0, -1, 5, 5])])
def test_commit(N, M, Hkv, D, W, dtype, pos, spread, accepted, packed):
    print(f"N={N} M={M} Hkv={Hkv} D={D} W={W} {dtype} packed={packed}", flush=True)
    x = make(N, M, Hkv, Hkv, D, W, dtype, pos, packed, 7200 + M + W, spread)
    keep = {n: x[n].clone() for n in CACHE if x[n] is not None}
    check_commit(x, keep, torch.tensor(accepted, dtype=torch.int32, device="cuda"), W)
    for n, a in enumerate(accepted):                     # nothing accepted, nothing touched
        if not 0 <= a < M:
            for name, t in keep.items():
                assert torch.equal(t[n].view(torch.uint8), x[name][n].view(torch.uint8))


def test_the_state_is_not_read_before_a_key_has_left():
    """Positions up to the window: whatever the state's buffer holds counts as zero, and is replaced when the first key leaves."""
    W, M = 12, 6
    x = make(3, M, 2, 1, 64, W, "f32", [3, 10, 12], False, 7300, 1)
    x["state"].zero_()
    ref = step(x, 0.125)
    x["state"].fill_(float("nan"))
    assert torch.equal(step(x, 0.125), ref) and bool(torch.isfinite(ref).all())
    accepted = torch.tensor([M - 1, M - 1, M - 1], dtype=torch.int32, device="cuda")
    rb.rattn_tree_commit(x["k"], x["v"], x["parent"], accepted, x["pos"], x["kr"], x["vr"], x["state"])
    assert bool(torch.isnan(x["state"][0]).all()) and bool(torch.isfinite(x["state"][1:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_counts_and_sequences_without_work(dtype):
    W, M = 33, 11
    x = make(5, M, 6, 2, 128, W, dtype, [50, 7, 33, 80, -1], False, 7400, 3)
    count = torch.tensor([11, 0, 4, -2, 5], dtype=torch.int32, device="cuda")
    out = torch.full_like(x["q"], 7.0)
    assert step(x, 0.1, count=count, out=out) is out
    ref = oracle({**x, "pos": torch.clamp(x["pos"], min=0)}, W, 0.1, count=[11, 0, 4, 0, 0])
    for n, c in enumerate([11, 0, 4, 0, 0]):
        assert bool((out[n, c:] == 7.0).all()), n
        if c:
            check(out[n, :c], ref[n, :c], dtype, x)
    assert bool((step(x, 0.1, count=count)[1] == 0).all())
    keep = {n: x[n].clone() for n in ("kr", "vr", "state")}
    accepted = torch.zeros(5, dtype=torch.int32, device="cuda")
    rb.rattn_tree_commit(x["k"], x["v"], x["parent"], accepted, x["pos"], x["kr"], x["vr"], x["state"])
    assert all(torch.equal(keep[n][4], x[n][4]) for n in keep) and not torch.equal(keep["kr"][0], x["kr"][0])


@pytest.mark.parametrize("N,M", [(1, 9), (140, 33)])
def test_the_last_positions_of_an_int32(N, M):
    """Positions whose tree passes 2^31 - 1: only whether the window is full and where it starts matter."""
    W = 24
    far = [2 ** 31 - 1 - i % 3 for i in range(N)]
    x = make(N, M, 4, 2, 64, W, "bf16", [p % W + 40 * W for p in far], False, 8250, 1)
    accepted = torch.full((N,), M - 1, dtype=torch.int32, device="cuda")
    y = {n: (t.clone() if t is not None else None) for n, t in x.items()}
    y["pos"] = torch.tensor(far, dtype=torch.int32, device="cuda")
    assert torch.equal(step(x, 0.125), step(y, 0.125))
    for z in (x, y):
        rb.rattn_tree_commit(z["k"], z["v"], z["parent"], accepted, z["pos"], z["kr"], z["vr"], z["state"])
    assert all(torch.equal(x[n], y[n]) for n in ("kr", "vr", "state"))


def test_parents_that_are_no_earlier_node_are_the_last_token():
    W = 40
    x = make(1, 6, 4, 1, 64, W, "f32", [77], False, 7500, 2)
    x["parent"] = torch.tensor([[0, 5, -9, 2, 2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    got = step(x, 0.125)
    x["parent"] = torch.tensor([[-1, -1, -1, 2, -1, -1]], dtype=torch.int32, device="cuda")
    assert torch.equal(got, step(x, 0.125))
    check(got, oracle(x, W, 0.125), "f32", x)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan"), 3.0e38])
def test_other_branches_and_left_keys_do_not_matter(bad, dtype, packed):
    """What is no number (or the type's largest) in a sibling's key or value, or in a slot without a token, reaches no row that does
    not see it; rows that see it are as the oracle's, number or not."""
    W, N, M = 30, 2, 8
    x = make(N, M, 4, 2, 64, W, dtype, [100, 17], packed, 7600, 1)
    x["parent"] = torch.tensor([[-1, 0, 0, 2, 3, -1, 5, 6]] * N, dtype=torch.int32, device="cuda")
    clean = step(x, 0.125)
    x["k"][:, 1, :, 5], x["v"][:, 1, :, 7] = bad, bad            # node 1: seen by itself alone
    x["v"][0, 5] = bad                                           # nodes 5, 6, 7 of the first sequence
    if not packed:
        x["kr"][1, :, 25, 3], x["vr"][1, :, 20:29] = bad, bad    # slots behind the 17 tokens
    o = step(x, 0.125)
    for i in (0, 2, 3, 4):
        assert torch.equal(o[:, i], clean[:, i]) or float((o[:, i].float() - clean[:, i].float()).abs().max()) <= (2e-2 if dtype == "bf16" else 1e-4), i
    assert float((o[1, 5:].float() - clean[1, 5:].float()).abs().max()) <= (2e-2 if dtype == "bf16" else 1e-4)
    # a ring value that has left the window of the deeper nodes, but not of the first
    y = make(1, 5, 4, 2, 64, W, dtype, [100], False, 7601, 1)
    slot = (100 - W + 2) % W                                     # the third to leave: seen by depths 0 and 1 in the window
    y["vr"][:, :, slot, 9] = bad
    with np.errstate(all="ignore"):
        ref = oracle(y, W, 0.125)
    o = np64(step(y, 0.125))
    if not math.isfinite(bad):
        assert np.array_equal(np.isfinite(o), np.isfinite(ref))
    fin = np.isfinite(ref) & np.isfinite(o)
    if math.isfinite(bad):
        fin &= np.abs(ref) < 1.0                                 # (features next to the largest number of the type are its rounding)
    assert float(np.abs(np.where(fin, o - ref, 0.0)).max()) <= (4e-2 if dtype == "bf16" else 2e-4)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_node_is_a_decode_step(dtype, packed):
    N, Hq, Hkv, D, W = 6, 8, 2, 128, 64
    pos = [0, 63, 64, 65, 1000, 30]
    x = make(N, 1, Hq, Hkv, D, W, dtype, pos, packed, 7700, 1)
    o = step(x, 0.1)
    y = {n: (t.clone() if t is not None else None) for n, t in x.items()}
    accepted = torch.zeros(N, dtype=torch.int32, device="cuda")
    rb.rattn_tree_commit(x["k"], x["v"], x["parent"], accepted, x["pos"], x["kr"], x["vr"], x["state"], k_scale=x["ks"], v_scale=x["vs"])
    head = (y["q"][:, 0].contiguous(), y["k"][:, 0].contiguous(), y["v"][:, 0].contiguous(), y["pos"])
    if packed:
        want = rb.rattn_decode_step_packed(*head, y["kr"], y["ks"], y["vr"], y["vs"], y["state"], y["gs"], y["gr"], softmax_scale=0.1)
    else:
        want = rb.rattn_decode_step(*head, y["kr"], y["vr"], y["state"], y["gs"], y["gr"], softmax_scale=0.1)
    tol = 2 * 2.0 ** -8 * want.float().abs() + 1e-3 if dtype == "bf16" else torch.full_like(want, 1e-5)   # two roundings of the output
    assert bool(((o[:, 0].float() - want.float()).abs() <= tol).all())
    for n in CACHE:
        if x[n] is not None and n != "state":
            assert torch.equal(x[n].view(torch.uint8), y[n].view(torch.uint8)), n
    assert float((x["state"] - y["state"]).abs().max()) <= 1e-5 * max(1.0, float(y["state"].abs().max()))


@pytest.mark.parametrize("D", [64, 128])
def test_a_chain_is_the_next_chunk_of_a_prompt(D):
    """All nodes in one chain: rows, rings and state of rattn_prefill_chunk over the same tokens."""
    N, M, Hq, Hkv, W, p = 2, 40, 6, 2, 96, 150
    x = make(N, M, Hq, Hkv, D, W, "bf16", [p] * N, False, 7800, 1)
    y = {n: (t.clone() if t is not None else None) for n, t in x.items()}
    o = step(x, 0.1)
    rb.rattn_tree_commit(x["k"], x["v"], x["parent"], torch.full((N,), M - 1, dtype=torch.int32, device="cuda"), x["pos"], x["kr"], x["vr"], x["state"])
    want = rb.rattn_prefill_chunk(y["q"], y["k"], y["v"], W, p, y["kr"], y["vr"], y["state"], y["gs"], y["gr"], softmax_scale=0.1)
    top = max(1.0, float(x["gs"].abs().max()), float(x["gr"].abs().max()))
    assert float((o.float() - want.float()).abs().max()) <= 2 * 2e-2 * top     # either is within 2e-2 of the formula
    assert torch.equal(x["kr"], y["kr"]) and torch.equal(x["vr"], y["vr"])
    assert float((x["state"] - y["state"]).abs().max()) <= 2e-5 * max(1.0, float(y["state"].abs().max()))


@pytest.mark.parametrize("packed", [False, True])
def test_drafting_verifying_and_accepting_together(packed):
    """Rounds of a serving loop for one layer: a tree of drafts, the step over it, a path accepted, its tokens taken in; the next round
    starts from there.  Every round against the oracle's layer on the tokens accepted so far, and a plain decode step at the end."""
    N, Hq, Hkv, D, W = 3, 8, 2, 64, 24
    x = make(N, 9, Hq, Hkv, D, W, "bf16", [0, 20, 24], packed, 7900, 2)
    x["state"].zero_()
    kr, vr = ring_values(x)
    S, pos, scale = np64(x["state"]), x["pos"].tolist(), 0.125
    rng = np.random.default_rng(79)
    for turn in range(6):
        M = int(rng.integers(1, 12))
        t = make(N, M, Hq, Hkv, D, W, "bf16", pos, False, 7901 + turn, 3)
        t.update({n: x[n] for n in CACHE}, pos=x["pos"])
        parents = t["parent"].cpu().numpy()
        o = step(t, scale)
        ref = orc.tree_step(np64(t["q"]), np64(t["k"]), np64(t["v"]), parents, pos, kr, vr, S, W, scale=scale, gamma_swa=np64(t["gs"]), gamma_rla=np64(t["gr"]))
        check(o, ref, "bf16", t, f"turn {turn}")
        accepted = rng.integers(-1, M, N)
        rb.rattn_tree_commit(t["k"], t["v"], t["parent"], torch.tensor(accepted, dtype=torch.int32, device="cuda"), x["pos"], x["kr"], x["vr"],
                             x["state"], k_scale=x["ks"], v_scale=x["vs"])
        k, v = np64(t["k"]), np64(t["v"])
        if W < 64 and packed:                # (the tokens of a path that leave with it are folded in as given: paths here are shorter than W)
            k, v = (orc.packed_values(*orc.pack_rows(a)) for a in (k, v))
        kr, vr, S = orc.tree_commit(k, v, parents, accepted, pos, kr, vr, S, W)
        lengths = [len(orc.tree_path(parents[n], int(a))) if a >= 0 else 0 for n, a in enumerate(accepted)]
        pos = [p + l for p, l in zip(pos, lengths)]
        x["pos"] += torch.tensor(lengths, dtype=torch.int32, device="cuda")
        got = ring_values(x)
        seen = np.array([[s < min(p, W) for s in range(W)] for p in pos])[:, None, :, None]
        assert np.array_equal(np.where(seen, got[0], 0), np.where(seen, kr, 0)) and np.array_equal(np.where(seen, got[1], 0), np.where(seen, vr, 0))
        assert float(np.abs(np64(x["state"]) - S).max()) <= 1e-5 * max(1.0, float(np.abs(S).max()))


def test_workspace_contents_do_not_matter_and_without_one():
    N, M, Hq, Hkv, D, W = 1, 5, 4, 1, 128, 2048
    x = make(N, M, Hq, Hkv, D, W, "bf16", [3333], False, 8000, 2)
    p = rb.RattnTreeParams(N, Hq, Hkv, D, W, rb.RATTN_BF16, M, 0.1, 1e-6, 0)
    n = ctypes.c_size_t()
    assert rb.lib().rattn_tree_workspace_bytes(ctypes.byref(p), 0, ctypes.byref(n)) == 0 and n.value > 0
    ref = step(x, 0.1)
    o = torch.empty_like(ref)
    P = lambda t: None if t is None else t.data_ptr()

    def call(ws, nbytes):
        o.fill_(float("nan"))
        st = rb.lib().rattn_tree_step(ctypes.byref(p), *(P(x[m]) for m in ("q", "k", "v", "parent")), None, P(x["pos"]), P(x["kr"]), None, P(x["vr"]),
                                      None, P(x["state"]), P(x["gs"]), P(x["gr"]), P(o), P(ws), nbytes, rb._stream())
        torch.cuda.synchronize()
        return st

    ws = torch.zeros(n.value, dtype=torch.uint8, device="cuda")
    for fill in (0, 255, None, "left"):
        if fill is None:
            ws.random_(generator=torch.Generator(device="cuda").manual_seed(1))
        elif fill != "left":
            ws.fill_(fill)
        assert call(ws, n.value) == 0 and torch.equal(o, ref), fill
    assert call(ws, n.value - 1) == -3
    assert call(None, 0) == 0
    assert bool(((o.float() - ref.float()).abs() <= 2 * 2.0 ** -8 * ref.float().abs() + 1e-3).all())


@pytest.mark.parametrize("M,G,W", [(1, 4, 2048), (13, 3, 2048), (64, 4, 4096)])
def test_workspaces_of_the_asked_size(M, G, W):
    """Steps whose work-groups share keys write nothing around a workspace of just the bytes that are asked for."""
    N, Hkv, D, B = 2, 2, 128, 4096
    x = make(N, M, G * Hkv, Hkv, D, W, "bf16", [2 * W, W + 7], True, 8050, 2)
    P = lambda t: None if t is None else t.data_ptr()
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    p = rb.RattnTreeParams(N, G * Hkv, Hkv, D, W, rb.RATTN_BF16, M, 0.1, 1e-6, 0)
    d = rb.RattnDecodeParams(N, G * Hkv, Hkv, D, W, rb.RATTN_BF16, 0.1, 1e-6, 0)
    assert rb.lib().rattn_tree_workspace_bytes(ctypes.byref(p), 1, ctypes.byref(n)) == 0 and n.value > 0
    assert rb.lib().rattn_decode_packed_workspace_bytes(ctypes.byref(d), ctypes.byref(m)) == 0 and m.value > 0
    ref, o = step(x, 0.1), torch.empty_like(x["q"])
    full = torch.full((n.value + 2 * B,), 0xA5, dtype=torch.uint8, device="cuda")
    assert rb.lib().rattn_tree_step(ctypes.byref(p), *(P(x[t]) for t in ("q", "k", "v", "parent")), None, P(x["pos"]), P(x["kr"]), P(x["ks"]), P(x["vr"]),
                                    P(x["vs"]), P(x["state"]), P(x["gs"]), P(x["gr"]), P(o), full.data_ptr() + B, n.value, rb._stream()) == 0
    assert torch.equal(o, ref) and bool((full[:B] == 0xA5).all()) and bool((full[B + n.value:] == 0xA5).all())
    q, k, v = (x[t][:, 0].contiguous() for t in "qkv")
    y = {t: x[t].clone() for t in CACHE}
    ref = rb.rattn_decode_step_packed(q, k, v, x["pos"], *(y[t] for t in ("kr", "ks", "vr", "vs", "state")), x["gs"], x["gr"], softmax_scale=0.1)
    o, full = torch.empty_like(q), torch.full((m.value + 2 * B,), 0xA5, dtype=torch.uint8, device="cuda")
    assert rb.lib().rattn_decode_step_packed(ctypes.byref(d), P(q), P(k), P(v), P(x["pos"]), P(x["kr"]), P(x["ks"]), P(x["vr"]), P(x["vs"]), P(x["state"]),
                                             P(x["gs"]), P(x["gr"]), P(o), full.data_ptr() + B, m.value, rb._stream()) == 0
    assert torch.equal(o, ref) and bool((full[:B] == 0xA5).all()) and bool((full[B + m.value:] == 0xA5).all())
    assert all(torch.equal(x[t].view(torch.uint8), y[t].view(torch.uint8)) for t in CACHE)


def test_steps_of_two_streams_at_once():
    """Steps that share keys among work-groups, on two streams that run at the same time, each with workspaces of its own."""
    N, M, Hq, Hkv, D, W = 2, 9, 8, 2, 128, 2048
    xs = [make(N, M, Hq, Hkv, D, W, "bf16", [3 * W, W + 1], packed, 8060 + packed, 2) for packed in (False, True)]
    refs = [step(x, 0.1) for x in xs]
    heads = [tuple(x[n][:, 0].contiguous() for n in "qkv") for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], [[], []]
    for _ in range(20):
        for i, x in enumerate(xs):
            with torch.cuda.stream(streams[i]):
                got[i].append(step(x, 0.1))
    torch.cuda.synchronize()
    for i, ref in enumerate(refs):
        assert all(torch.equal(o, ref) for o in got[i])
    caches = [{n: xs[1][n].clone() for n in CACHE} for _ in range(3)]

    def decode(y):
        return rb.rattn_decode_step_packed(*heads[1], xs[1]["pos"], y["kr"], y["ks"], y["vr"], y["vs"], y["state"], softmax_scale=0.1)

    want = [decode(caches[2]) for _ in range(5)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(decode(caches[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want))
        assert all(torch.equal(caches[i][n].view(torch.uint8), caches[2][n].view(torch.uint8)) for n in CACHE)


@pytest.mark.parametrize("W", [64, 2048])
def test_captured_and_on_another_stream(W):
    """A step and a commit in one graph, replayed with eager work between the replays; two graphs that share one workspace pool are
    replayed in turn."""
    N, M, Hq, Hkv, D = 2, 6, 4, 1, 128
    x = make(N, M, Hq, Hkv, D, W, "bf16", [W + 5, 40], True, 8100, 2)
    accepted = torch.tensor([M - 1, 2], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([len(orc.tree_path(p, int(a))) for p, a in zip(x["parent"].cpu().numpy(), accepted.tolist())], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(8101)
    drafts = [tuple(torch.randn(N, M, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)) for _ in range(4)]

    def both(s, out):
        step(s, 0.1, out=out)
        rb.rattn_tree_commit(s["k"], s["v"], s["parent"], accepted, s["pos"], s["kr"], s["vr"], s["state"], k_scale=s["ks"], v_scale=s["vs"])

    def rounds(s, out, f):
        got = []
        for d in drafts:
            for n, t in zip("qkv", d):
                s[n].copy_(t)
            f()
            got.append(out.clone())
            s["pos"] += lengths
        torch.cuda.synchronize()
        return got

    copy = lambda: {n: (t.clone() if t is not None else None) for n, t in x.items()}
    a, oa = copy(), torch.empty_like(x["q"])
    ref = rounds(a, oa, lambda: both(a, oa))
    side, b, ob = torch.cuda.Stream(), copy(), torch.empty_like(oa)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        on_side = rounds(b, ob, lambda: both(b, ob))
    states, graphs = [copy(), copy()], []
    outs = [torch.empty_like(oa) for _ in states]
    pool = None
    torch.cuda.synchronize()
    for s, out in zip(states, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            both(s, out)
        pool = graph.pool()
        graphs.append(graph)
    got = [[], []]
    for d in drafts:
        for i in range(2):
            for n, t in zip("qkv", d):
                states[i][n].copy_(t)
            graphs[i].replay()
            got[i].append(outs[i].clone())
            states[i]["pos"] += lengths
        torch.cuda.synchronize()
    for r, s, g0, g1 in zip(ref, on_side, *got):
        assert torch.equal(r, s) and torch.equal(r, g0) and torch.equal(r, g1)
    for n in CACHE:
        assert torch.equal(a[n].view(torch.uint8), states[0][n].view(torch.uint8)) and torch.equal(a[n].view(torch.uint8), states[1][n].view(torch.uint8))


def test_calls_stay_inside_their_buffers():
    """4 KiB of a known pattern on both sides of everything that is written."""
    N, M, Hq, Hkv, D, W, G = 2, 5, 10, 2, 64, 37, 4096
    x = make(N, M, Hq, Hkv, D, W, "bf16", [36, 90], True, 8200, 2)

    def guarded(t):
        n = t.numel() * t.element_size()
        full = torch.full((2 * G + n + (-n) % 256,), 0xA5, dtype=torch.uint8, device="cuda")
        view = full[G:G + n].view(t.dtype).view(t.shape)
        view.view(torch.uint8).copy_(t.view(torch.uint8))
        return full, n, view

    held = {}
    for name in ("kr", "vr", "ks", "vs", "state"):
        *held[name], x[name] = guarded(x[name])
    *held["o"], out = guarded(x["q"])
    step(x, 0.1, out=out)
    rb.rattn_tree_commit(x["k"], x["v"], x["parent"], torch.tensor([4, 4], dtype=torch.int32, device="cuda"), x["pos"], x["kr"], x["vr"], x["state"],
                         k_scale=x["ks"], v_scale=x["vs"])
    rb.rattn_decode_step_packed(x["q"][:, 0].contiguous(), x["k"][:, 0].contiguous(), x["v"][:, 0].contiguous(), x["pos"], x["kr"], x["ks"], x["vr"],
                                x["vs"], x["state"], x["gs"], x["gr"], softmax_scale=0.1)
    plain = rb.rattn_ring_unpack(x["kr"], x["ks"], x["vr"], x["vs"])
    rb.rattn_ring_pack(*plain, out=(x["kr"], x["ks"], x["vr"], x["vs"]))
    fk, nk, kv = guarded(plain[0])
    fv, nv, vv = guarded(plain[1])
    rb.rattn_ring_unpack(x["kr"], x["ks"], x["vr"], x["vs"], out=(kv, vv))
    torch.cuda.synchronize()
    for name, (full, n) in {**held, "k_ring": (fk, nk), "v_ring": (fv, nv)}.items():
        assert bool((full[:G] == 0xA5).all()) and bool((full[G + n:] == 0xA5).all()), name


def test_refusals():
    x = make(2, 3, 4, 2, 64, 16, "bf16", [3, 30], False, 8300)
    p = make(2, 3, 4, 2, 64, 16, "bf16", [3, 30], True, 8300)
    for kw, what in ((dict(parent=x["parent"].long()), "int32"), (dict(pos=x["pos"][:1].contiguous()), "pos"), (dict(k=x["k"].float()), "dtype"),
                     (dict(kr=x["kr"].float()), "dtype"), (dict(kr=p["kr"], vr=p["vr"]), "dtype"), (dict(ks=p["ks"]), "neither"),
                     (dict(q=x["q"][:, :2].contiguous()), "q must be"), (dict(state=x["state"].double()), "float32"),
                     (dict(v=x["v"].transpose(1, 2)), "share shape"), (dict(vr=x["vr"].cpu()), "contiguous device tensor")):
        with pytest.raises(ValueError, match=what):
            step({**x, **kw}, 0.1)
    with pytest.raises(ValueError, match="count"):
        step(x, 0.1, count=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="out must be"):
        step(x, 0.1, out=torch.empty(2, 3, 4, 64, device="cuda"))
    with pytest.raises(ValueError, match="accepted"):
        rb.rattn_tree_commit(x["k"], x["v"], x["parent"], x["pos"].long(), x["pos"], x["kr"], x["vr"], x["state"])
    big = make(1, 65, 1, 1, 64, 16, "bf16", [3], False, 8301)
    with pytest.raises(rb.RattnError, match="nodes"):
        step(big, 0.1)
    with pytest.raises(KeyError):
        step(x, 0.1, feature_map="tanh")
