"""Drafted tokens over packed rings and the packed decode steps that would have brought them one by one.  A node sees its ancestors as
they are given, and a commit folds what leaves at once (paths longer than the window) as given; a decode step stores a token in 8
bits, and the steps after it see that.  So the two agree where packing keeps the drafts' keys and values, rings always to the bit, and
the state differs by the rounding of just those tokens that never had a slot."""
import pytest
import torch

from paper_2506_15545_amd import binding as rb
from test_gpu_tree import CACHE, DT, make, step

pytestmark = pytest.mark.gpu
PACKED = ("kr", "ks", "vr", "vs")


def kept_by_packing(k, v):
    """k, v [N,M,Hkv,D] as they are read back from 8 bits."""
    return rb.rattn_ring_unpack(*rb.rattn_ring_pack(k, v), k.dtype)


def copy(x):
    return {n: (t.clone() if torch.is_tensor(t) else t) for n, t in x.items()}


def commit(x, k, v, parent, last):
    accepted = torch.full((k.shape[0],), last, dtype=torch.int32, device="cuda")
    rb.rattn_tree_commit(k, v, parent, accepted, x["pos"], x["kr"], x["vr"], x["state"], k_scale=x["ks"], v_scale=x["vs"])


def one_by_one(x, scale):
    """The chain's tokens through packed decode steps, on x's cache; their outputs [N,M,Hq,D]."""
    out = []
    for d in range(x["k"].shape[1]):
        q, k, v = (x[n][:, d].contiguous() for n in "qkv")
        out.append(rb.rattn_decode_step_packed(q, k, v, x["pos"] + d, *(x[n] for n in PACKED), x["state"], x["gs"], x["gr"], softmax_scale=scale))
    return torch.stack(out, 1)


def same_rings(x, y):
    return all(torch.equal(x[n].view(torch.uint8), y[n].view(torch.uint8)) for n in PACKED)


def close_states(a, b):
    return float((a.double() - b.double()).abs().max()) <= 2e-5 * max(1.0, float(b.abs().max()))   # either 1e-5 off the formula


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,W,pos", [(9, 40, [100, 3, 38]), (25, 10, [0, 7, 200]), (64, 33, [33, 500])])
def test_drafts_that_packing_keeps_are_packed_decode_steps(M, W, pos, dtype, D):
    """Outputs: either is within the layer's bar of the formula (fp32 1e-4 of unit scale); bf16: two-term operands leave 2^-14 of a row
    whose largest feature is below 12 gains, and either is rounded (2^-8 of its value at most)."""
    x = make(len(pos), M, 8, 2, D, W, dtype, pos, True, 8800 + M, 1)
    x["k"], x["v"] = kept_by_packing(x["k"], x["v"])
    y, scale = copy(x), D ** -0.5
    o, want = step(x, scale), one_by_one(y, scale)
    top = max(1.0, float(x["gs"].abs().max()), float(x["gr"].abs().max()))
    bar = 2 * 2.0 ** -8 * want.float().abs() + 2 * 2.0 ** -14 * 12 * top if dtype == "bf16" else torch.full_like(want, 2e-4 * top)
    assert bool(((o.float() - want.float()).abs() <= bar).all())
    commit(x, x["k"], x["v"], x["parent"], M - 1)
    assert same_rings(x, y) and close_states(x["state"], y["state"])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("first,second", [(25, 0), (12, 13), (9, 6), (3, 40)])
def test_a_commit_folds_tokens_without_a_slot_as_given(first, second, dtype, D):
    W, pos, M = 10, [0, 7, 10, 200], first + second
    x = make(len(pos), M, 4, 2, D, W, dtype, pos, True, 8900 + first, 1)
    k8, v8 = kept_by_packing(x["k"], x["v"])
    y = copy(x)
    one_by_one(y, 0.1)
    chain = lambda n: (torch.arange(n, dtype=torch.int32, device="cuda") - 1).expand(len(pos), n).contiguous()
    start = 0
    never = []                                   # tokens that left in the commit that brought them
    for n in (first, second):
        if n:
            commit(x, x["k"][:, start:start + n].contiguous(), x["v"][:, start:start + n].contiguous(), chain(n), n - 1)
            x["pos"] += n
            never += range(start, start + max(0, n - W))
            start += n
    phi = lambda t: torch.softmax(t.double(), -1)
    fold = lambda k, v: torch.einsum("nmhf,nmhd->nhfd", phi(k[:, never]).cpu(), v[:, never].double().cpu()).cuda()
    assert same_rings(x, y)
    assert close_states(x["state"], y["state"] + fold(x["k"], x["v"]) - fold(k8, v8))
