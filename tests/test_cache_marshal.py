"""The native argument marshalling of packed rings and trees: what it takes, what it leaves to the Python path, and that both give the
same; without the extension everything goes through Python."""
import sys

import pytest
import torch

import paper_2506_15545_amd
from paper_2506_15545_amd import binding as rb

CALLS = ("ring_pack", "ring_unpack", "decode_step_packed", "tree_step", "tree_commit")


@pytest.fixture
def python_only(monkeypatch):
    native = rb._Native()
    native.__dict__.update(dict.fromkeys(CALLS, rb._no_native))
    return lambda: monkeypatch.setattr(rb, "_native", native)


def test_without_the_extension(monkeypatch):
    monkeypatch.setitem(sys.modules, "paper_2506_15545_amd._marshal", None)   # importing it raises ImportError
    monkeypatch.delattr(paper_2506_15545_amd, "_marshal", raising=False)
    monkeypatch.setattr(rb, "_native", rb._Native())
    k = torch.zeros(1, 1, 4, 64)
    with pytest.raises(ValueError, match="contiguous device tensor"):
        rb.rattn_ring_pack(k, k)
    assert rb._native.tree_step is rb._no_native


def test_host_tensors_and_odd_arguments_are_left_to_python():
    k, t = torch.zeros(1, 1, 4, 64), torch.zeros(1, dtype=torch.int32)
    n = rb._native
    assert n.ring_pack(k, k, None) is None and n.ring_pack(None, 3, None) is None
    assert n.ring_unpack(k, k, k, k, (k, k)) is None and n.ring_unpack(k, k, k, k, None) is None
    assert n.decode_step_packed(*[k] * 9, None, None, 1.0, 1e-6, None, "softmax") is None
    assert n.tree_step(*[k] * 8, None, None, 1.0, 1e-6, None, None, None, None, "softmax") is None
    assert n.tree_commit(*[k] * 8, None, None, "softmax") is None
    with pytest.raises(TypeError):
        n.tree_commit(k)


def tensors(dtype, N=2, M=4, Hq=4, Hkv=2, D=64, W=16):
    g = torch.Generator().manual_seed(8500)
    r = lambda *s, dt=dtype: torch.randn(*s, generator=g).to(dt).cuda()
    x = dict(q=r(N, M, Hq, D), k=r(N, M, Hkv, D), v=r(N, M, Hkv, D), kr=r(N, Hkv, W, D), vr=r(N, Hkv, W, D), state=r(N, Hkv, D, D, dt=torch.float32),
             gs=r(Hq, D, dt=torch.float32), gr=r(Hq, D, dt=torch.float32))
    x["parent"] = (torch.arange(M, dtype=torch.int32) - 1).repeat(N, 1).contiguous().cuda()
    x["pos"], x["count"], x["accepted"] = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([3, 30], [4, 2], [1, 3]))
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_both_ways_give_the_same(dtype, python_only):
    def all_calls():
        x = tensors(dtype)
        got = list(rb.rattn_ring_pack(x["kr"], x["vr"]))
        kc, ks, vc, vs = (t.clone() for t in got)
        got += rb.rattn_ring_unpack(kc, ks, vc, vs, dtype)
        out = torch.zeros_like(x["q"])
        for scales, rings in (({}, (x["kr"], x["vr"])), (dict(k_scale=ks, v_scale=vs), (kc, vc))):
            a = (x["q"], x["k"], x["v"], x["parent"], x["pos"], *rings, x["state"])
            got += [rb.rattn_tree_step(*a, **scales), rb.rattn_tree_step(*a, x["gs"], x["gr"], 0.5, 1e-5, count=x["count"], feature_map="relu", **scales)]
            assert rb.rattn_tree_step(*a, count=x["count"], out=out, **scales) is out
            got.append(out.clone())
            S = x["state"].clone()
            assert rb.rattn_tree_commit(x["k"], x["v"], x["parent"], x["accepted"], x["pos"], *rings, S, **scales) is None
            got += [S, *(t.clone() for t in rings)]
        S = x["state"].clone()
        one = (x["q"][:, 0].contiguous(), x["k"][:, 0].contiguous(), x["v"][:, 0].contiguous(), x["pos"], kc, ks, vc, vs, S)
        got += [rb.rattn_decode_step_packed(*one), rb.rattn_decode_step_packed(*one, x["gs"], x["gr"], softmax_scale=0.5, feature_map="identity"),
                S, kc, ks, vc, vs]
        torch.cuda.synchronize()
        return got

    a = all_calls()
    assert rb._native.tree_step is not rb._no_native
    python_only()
    b = all_calls()
    assert len(a) == len(b)
    for i, (x, y) in enumerate(zip(a, b)):
        assert x.dtype == y.dtype and torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i


@pytest.mark.gpu
def test_what_the_native_path_takes_and_leaves():
    x = tensors(torch.bfloat16)
    n = rb._native
    kc, ks, vc, vs = rb.rattn_ring_pack(x["kr"], x["vr"])
    step = lambda **kw: n.tree_step(*({**x, **kw}[m] for m in ("q", "k", "v", "parent", "pos", "kr", "vr", "state")), None, None,
                                    kw.get("scale", 1.0), 1e-6, None, kw.get("ks"), kw.get("vs"), None, "softmax")
    assert isinstance(step(), torch.Tensor) and isinstance(step(kr=kc, vr=vc, ks=ks, vs=vs), torch.Tensor)
    for kw in (dict(q=x["q"].float()), dict(kr=kc), dict(ks=ks, vs=vs), dict(kr=kc, vr=vc, ks=ks), dict(scale=1), dict(pos=x["pos"].long()),
               dict(k=x["k"].transpose(1, 2)), dict(parent=x["parent"][:1].contiguous()), dict(state=x["state"].bfloat16())):
        assert step(**kw) is None, kw.keys()
    assert step(scale=0.0) == -1                       # the library's refusal, as a status
    with pytest.raises(rb.RattnError):
        rb.rattn_tree_step(*(x[m] for m in ("q", "k", "v", "parent", "pos", "kr", "vr", "state")), softmax_scale=0.0)
    assert isinstance(rb.rattn_tree_step(*(x[m] for m in ("q", "k", "v", "parent", "pos", "kr", "vr", "state")), softmax_scale=1), torch.Tensor)
    assert n.tree_commit(x["k"], x["v"], x["parent"], x["accepted"], x["pos"], x["kr"], x["vr"], x["state"], None, None, "softmax") is True
