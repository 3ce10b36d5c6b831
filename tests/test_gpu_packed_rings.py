"""Packed rings: packing and unpacking to the bit, and the decode step over them, against the fp64 oracle."""
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
NAMES = ("q", "k_new", "v_new", "pos", "kc", "ks", "vc", "vs", "state")


def values(codes, scales):
    return orc.packed_values(np64(codes), np64(scales))


def awkward_rows(N, Hkv, W, D, dtype, seed):
    """Rows of normal numbers at very different scales, with ties, limits, zeros and what is no number among them."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, Hkv, W, D, generator=g) * torch.exp(20 * torch.randn(N, Hkv, W, 1, generator=g))
    rows = x.view(-1, D)
    tie = (8 + torch.arange(D) % 8 + 0.5) * 2.0 ** (torch.arange(D) // 8 % 6 - 3)      # halfway between two numbers
    for r, row in enumerate([torch.zeros(D), -torch.zeros(D), tie, -tie, torch.full((D,), 448.0), torch.full((D,), 449.0),
                             torch.linspace(220, 228, D), torch.linspace(-455, 470, D), torch.full((D,), 3.0e38), torch.full((D,), 1e-38),
                             torch.full((D,), 2.0 ** -130), 2.0 ** -torch.arange(D).float()]):
        if r < len(rows):
            rows[r] = row
    if len(rows) > 14:
        rows[12, 3], rows[12, 40], rows[13, 5], rows[14] = float("inf"), -float("inf"), float("nan"), float("nan")
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,Hkv,W,D", [(1, 1, 1, 64), (2, 3, 5, 128), (1, 2, 333, 64), (3, 1, 1030, 128)])
def test_pack_and_unpack(N, Hkv, W, D, dtype):
    k, v = awkward_rows(N, Hkv, W, D, dtype, 1), awkward_rows(N, Hkv, W, D, dtype, 2)
    kc, ks, vc, vs = rb.rattn_ring_pack(k.cuda(), v.cuda())
    for x, c, s in ((k, kc, ks), (v, vc, vs)):
        codes, scales = orc.pack_rows(np64(x))
        assert np.array_equal(np64(s), scales)
        assert np.array_equal(np64(c), codes, equal_nan=True)
        for out in DT.values():
            got, _ = rb.rattn_ring_unpack(c, s, vc, vs, out)
            want = codes * np.repeat(scales, 32, -1)
            # both types hold the values: fp32 from 2^-149 on, bf16 from 2^-133 on, where half a step is 2^-134
            tiny = 2.0 ** -150 if out == torch.float32 else 2.0 ** -134
            err = np.abs(np64(got) - want)
            assert np.array_equal(np.isnan(np64(got)), np.isnan(want)) and float(np.nanmax(err, initial=0.0)) <= tiny
    # packing what was unpacked stands for the same values; given tensors are filled
    k2, v2 = rb.rattn_ring_unpack(kc, ks, vc, vs, torch.float32)
    out = tuple(torch.zeros_like(t.view(torch.uint8)).view(t.dtype) for t in (kc, ks, vc, vs))
    assert rb.rattn_ring_pack(k2, v2, out=out) is out
    assert np.array_equal(values(out[0], out[1]), values(kc, ks), equal_nan=True)
    assert np.array_equal(values(out[2], out[3]), values(vc, vs), equal_nan=True)
    given = (torch.zeros_like(k2), torch.zeros_like(v2))
    assert rb.rattn_ring_unpack(*out, torch.float32, out=given)[0] is given[0] and torch.equal(given[1].nan_to_num(), v2.nan_to_num())


def step_inputs(N, Hq, Hkv, D, W, dtype, pos, seed):
    cfg = synth.DecodeConfig("packed", N, Hq, Hkv, D, W, dtype, seed, 0, max(pos), 1.0 / math.sqrt(D))
    d = synth.make_decode_inputs(cfg, pos=pos)
    g = torch.Generator().manual_seed(seed + 1)
    gains = tuple(1.0 + 0.25 * torch.randn(Hq, D, generator=g) for _ in range(2))
    x = {n: t.cuda() for n, t in d.items()}
    x["kc"], x["ks"], x["vc"], x["vs"] = rb.rattn_ring_pack(x.pop("k_ring"), x.pop("v_ring"))
    return x, tuple(t.cuda() for t in gains), cfg.scale


def oracle_step(x, gains, scale, W, phi="softmax"):
    return orc.decode_step(np64(x["q"]), np64(x["k_new"]), np64(x["v_new"]), x["pos"].tolist(), values(x["kc"], x["ks"]),
                           values(x["vc"], x["vs"]), np64(x["state"]), W, scale=scale, gamma_swa=np64(gains[0]),
                           gamma_rla=np64(gains[1]), feature_map=phi)


def check_out(o, ref, dtype, gains):
    top = max(1.0, float(gains[0].abs().max()), float(gains[1].abs().max()))
    if dtype == "bf16":
        pm.assert_out_bf16(np64(o), ref, gain_scale=top)
    else:
        err = float(np.abs(np64(o) - ref).max())
        print(f"o: max-abs {err:.2e}", flush=True)
        assert err <= 1e-4 * top


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("N,Hq,Hkv,W,pos", [
    (1, 1, 1, 1, [0]), (3, 2, 1, 1, [1, 2, 9]), (4, 4, 2, 3, [0, 2, 3, 40]), (5, 6, 2, 37, [0, 1, 36, 37, 500]),
    (2, 16, 1, 100, [99, 100]), (2, 20, 1, 130, [64, 1000]),               # one pass over the rings, two
    (3, 34, 2, 65, [5, 65, 66]), (2, 4, 1, 4097, [4096, 9000]),            # three; shared rings
    (1, 3, 1, 8200, [300]), (40, 8, 8, 64, [30 * i for i in range(40)])])
def test_decode_step(N, Hq, Hkv, D, W, dtype, pos):
    print(f"N={N} Hq={Hq} Hkv={Hkv} D={D} W={W} {dtype}", flush=True)
    x, gains, scale = step_inputs(N, Hq, Hkv, D, W, dtype, pos, 6100 + W + N)
    o_ref, kr, vr, S = oracle_step(x, gains, scale, W)
    before = {n: np64(x[n]) for n in ("kc", "ks", "vc", "vs")}
    o = rb.rattn_decode_step_packed(*(x[n] for n in NAMES), *gains, softmax_scale=scale)
    check_out(o, o_ref, dtype, gains)
    assert float(np.abs(np64(x["state"]) - S).max()) <= 1e-5 * max(1.0, float(np.abs(S).max()))
    # the new token's row to the bit, every other one as it was
    for c, s, new in (("kc", "ks", "k_new"), ("vc", "vs", "v_new")):
        codes, scales = orc.pack_rows(np64(x[new]))
        for n, p in enumerate(pos):
            before[c][n, :, p % W], before[s][n, :, p % W] = codes[n], scales[n]
        assert np.array_equal(np64(x[c]), before[c]) and np.array_equal(np64(x[s]), before[s])


@pytest.mark.parametrize("phi", ["relu", "identity"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_feature_maps(phi, dtype):
    W = 40
    x, gains, scale = step_inputs(3, 6, 2, 64, W, dtype, [7, 40, 99], 6200)
    o_ref, _, _, S = oracle_step(x, gains, scale, W, phi)
    o = rb.rattn_decode_step_packed(*(x[n] for n in NAMES), *gains, softmax_scale=scale, feature_map=phi)
    check_out(o, o_ref, dtype, gains)
    assert float(np.abs(np64(x["state"]) - S).max()) <= 1e-5 * max(1.0, float(np.abs(S).max()))


def test_rounding_of_the_rings_is_all_that_differs_from_the_plain_step():
    """The same step over the unpacked rings: bf16 outputs within two roundings of bf16 of each other."""
    W = 512
    x, gains, scale = step_inputs(8, 32, 8, 128, W, "bf16", [100, 511, 512, 513, 2000, 0, 1, 30000], 6300)
    kr, vr = rb.rattn_ring_unpack(x["kc"], x["ks"], x["vc"], x["vs"])
    y = {n: t.clone() for n, t in x.items()}
    o1 = rb.rattn_decode_step_packed(*(x[n] for n in NAMES), *gains, softmax_scale=scale)
    o2 = rb.rattn_decode_step(y["q"], y["k_new"], y["v_new"], y["pos"], kr, vr, y["state"], *gains, softmax_scale=scale)
    assert torch.equal(x["state"], y["state"])
    assert bool(((o1.float() - o2.float()).abs() <= 2 * 2.0 ** -8 * o2.float().abs() + 1e-3).all())


def test_what_is_no_number_stays_with_its_token():
    """A value that is infinite (stored as NaN) in the slot that the new token takes: it is in the state by then, but not among the
    keys of the window.  With the ReLU map and a key without positive features nothing but 0 times it reaches the state."""
    W, N = 48, 2
    x, gains, scale = step_inputs(N, 4, 1, 64, W, "bf16", [60, 20], 6400)
    kr, vr = rb.rattn_ring_unpack(x["kc"], x["ks"], x["vc"], x["vs"])
    vr[1, 0, 30] = float("inf")                       # a slot that holds no token yet
    x["kc"], x["ks"], x["vc"], x["vs"] = rb.rattn_ring_pack(kr, vr)
    assert bool(torch.isnan(x["vc"][1, 0, 30].float()).all())
    o_ref, _, _, _ = orc.decode_step(np64(x["q"]), np64(x["k_new"]), np64(x["v_new"]), [60, 20], values(x["kc"], x["ks"]),
                                     values(x["vc"], x["vs"]), np64(x["state"]), W, scale=scale, gamma_swa=np64(gains[0]), gamma_rla=np64(gains[1]))
    o = rb.rattn_decode_step_packed(*(x[n] for n in NAMES), *gains, softmax_scale=scale)
    assert bool(torch.isfinite(o).all())
    check_out(o, o_ref, "bf16", gains)


def test_a_chain_of_steps_on_another_stream_and_captured():
    """Steps that wrap the window, eagerly, on a side stream and as replays of one graph with eager work between them: the same bits;
    the rings are shared by work-groups that meet in the workspace."""
    N, Hq, Hkv, D, W, steps = 2, 4, 1, 128, 4096, 5
    x, gains, scale = step_inputs(N, Hq, Hkv, D, W, "bf16", [4093, 1], 6500)
    g = torch.Generator(device="cuda").manual_seed(6501)
    new = [tuple(torch.randn(N, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv)) for _ in range(steps)]

    def run(step, state):
        outs = []
        for i in range(steps):
            for n, t in zip(("q", "k_new", "v_new"), new[i]):
                state[n].copy_(t)
            outs.append(step(state).clone())
            state["pos"] += 1
        torch.cuda.synchronize()
        return outs

    eager = lambda s: rb.rattn_decode_step_packed(*(s[n] for n in NAMES), *gains, softmax_scale=scale)
    a = {n: t.clone() for n, t in x.items()}
    ref = run(eager, a)
    b = {n: t.clone() for n, t in x.items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out_side = run(eager, b)
    c = {n: t.clone() for n, t in x.items()}
    out = torch.empty_like(c["q"])
    warm = {n: t.clone() for n, t in x.items()}
    with torch.cuda.stream(side):
        rb.rattn_decode_step_packed(*(warm[n] for n in NAMES), *gains, softmax_scale=scale)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rb.rattn_decode_step_packed(*(c[n] for n in NAMES), *gains, softmax_scale=scale, out=out)

    def replay(s):
        graph.replay()
        torch.cuda.synchronize()
        return out

    out_graph = run(replay, c)
    for i in range(steps):
        assert torch.equal(ref[i], out_side[i]) and torch.equal(ref[i], out_graph[i]), i
    for n in ("kc", "vc", "ks", "vs"):
        assert torch.equal(a[n].view(torch.uint8), b[n].view(torch.uint8)) and torch.equal(a[n].view(torch.uint8), c[n].view(torch.uint8))
    assert torch.equal(a["state"], c["state"])


def test_hand_over_from_a_prompt():
    """A prompt's rings packed, then decode steps: the oracle's steps over the packed values."""
    B, T, Hq, Hkv, D, W = 2, 150, 4, 2, 64, 100
    x = synth.make_random_layer(B, T, Hq, Hkv, D, "bf16", 6600)
    k, v = x["k"].cuda(), x["v"].cuda()
    kr, vr, S = rb.rattn_prefill_export(k, v, W)
    packed = rb.rattn_ring_pack(kr, vr)
    scale, pos = D ** -0.5, torch.full((B,), T, dtype=torch.int32, device="cuda")
    rk, rv, rS = values(*packed[:2]), values(*packed[2:]), np64(S)
    g = torch.Generator(device="cuda").manual_seed(6601)
    for i in range(3):
        q, kn, vn = (torch.randn(B, h, D, generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
        o_ref, rk, rv, rS = orc.decode_step(np64(q), np64(kn), np64(vn), [T + i] * B, rk, rv, rS, W, scale=scale)
        for ring, new in ((rk, kn), (rv, vn)):       # what is stored of the new token
            ring[:, :, (T + i) % W] = orc.packed_values(*orc.pack_rows(np64(new)))
        o = rb.rattn_decode_step_packed(q, kn, vn, pos, *packed, S, softmax_scale=scale)
        pos += 1
        pm.assert_out_bf16(np64(o), o_ref)
        assert float(np.abs(np64(S) - rS).max()) <= 1e-5 * max(1.0, float(np.abs(rS).max()))


def test_refusals():
    x, gains, scale = step_inputs(2, 4, 2, 64, 16, "bf16", [3, 30], 6700)
    call = lambda **kw: rb.rattn_decode_step_packed(*({**x, **kw}[n] for n in NAMES))
    for kw, what in ((dict(kc=x["kc"].view(torch.uint8)), "float8_e4m3fn"), (dict(ks=x["ks"].view(torch.uint8)), "float8_e8m0fnu"),
                     (dict(vs=x["vs"][..., :1].contiguous()), "v_scale"), (dict(pos=x["pos"].long()), "int32"),
                     (dict(state=x["state"].bfloat16()), "float32"), (dict(k_new=x["k_new"].float()), "share dtype"),
                     (dict(q=x["q"].transpose(0, 1)), "contiguous"), (dict(pos=x["pos"].cpu()), "device"),
                     (dict(v_new=x["v_new"][:1].contiguous()), "shapes")):
        with pytest.raises(ValueError, match=what):
            call(**kw)
    with pytest.raises(ValueError, match="out must be"):
        rb.rattn_decode_step_packed(*(x[n] for n in NAMES), out=torch.empty(2, 4, 64, device="cuda"))
    with pytest.raises(rb.RattnError):
        rb.rattn_decode_step_packed(*(x[n] for n in NAMES), rms_eps=0.0)
    k = torch.zeros(1, 1, 4, 64, device="cuda")
    with pytest.raises(ValueError):
        rb.rattn_ring_pack(k, k.bfloat16())
    with pytest.raises(ValueError):
        rb.rattn_ring_pack(k.half(), k.half())
    with pytest.raises(rb.RattnError):
        z = torch.zeros(1, 1, 4, 96, device="cuda")
        rb.rattn_ring_pack(z, z)
    with pytest.raises(ValueError, match="dtype"):
        rb.rattn_ring_unpack(x["kc"], x["ks"], x["vc"], x["vs"], torch.float16)
