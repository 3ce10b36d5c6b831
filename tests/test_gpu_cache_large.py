"""Caches whose offsets pass 32 bits: many sequences, and one ring alone.  What the calls find there is compared with the same calls on
a copy of the sequence by itself, or with the formula in fp64 over the whole ring."""
import pytest
import torch

from paper_2506_15545_amd import binding as rb

pytestmark = pytest.mark.gpu
SCALE, EPS = 0.09, 1e-6


def cache(N, Hkv, W, D, dtype, packed, seed):
    """Random rings (the same few thousand rows in turn, so that they are quick to make) and state."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=dtype: torch.randn(*s, generator=g, device="cuda").to(dt)
    some = [r(1, 1, 4099, D) for _ in range(2)]     # (a prime: rows of different sequences differ)
    rows = N * Hkv * W
    if packed:
        some = rb.rattn_ring_pack(*some)
    x = {}
    for name, t in zip(("kr", "ks", "vr", "vs") if packed else ("kr", "vr"), some):
        bits = t.view(torch.uint8).view(4099, -1)
        full = torch.empty(rows, bits.shape[1], dtype=torch.uint8, device="cuda")
        n = rows // 4099 * 4099
        full[:n].view(-1, 4099, bits.shape[1]).copy_(bits)
        full[n:].copy_(bits[: rows - n])
        x[name] = full.view(t.dtype).view(N, Hkv, W, t.shape[-1])
    x["state"] = 0.1 * r(N, Hkv, D, D, dt=torch.float32)
    return x, r


def alone(x, n):
    return {name: t[n:n + 1].clone() for name, t in x.items()}


def same(a, b):
    return all(torch.equal(a[n].view(torch.uint8), b[n].view(torch.uint8)) for n in b)


@pytest.mark.parametrize("dtype,packed", [(torch.bfloat16, False), (torch.bfloat16, True), (torch.float32, False)])
def test_many_sequences(dtype, packed):
    """Rings of 2.2e9 features and more: the last sequence begins behind 2^31 of them, behind 2^32 bytes where a feature has two."""
    N, Hkv, W, D, M = 530 if not packed else 1100, 8, 4096, 128, 3
    x, r = cache(N, Hkv, W, D, dtype, packed, 8950)
    q, k, v = r(N, M, Hkv, D), r(N, M, Hkv, D), r(N, M, Hkv, D)
    pos = torch.full((N,), W + 77, dtype=torch.int32, device="cuda")
    parent = torch.tensor([[-1, 0, 0]], dtype=torch.int32, device="cuda").repeat(N, 1)
    accepted = torch.full((N,), 2, dtype=torch.int32, device="cuda")
    scales = lambda c: dict(k_scale=c.get("ks"), v_scale=c.get("vs"))
    tree = lambda c, i: rb.rattn_tree_step(q[i], k[i], v[i], parent[i], pos[i], c["kr"], c["vr"], c["state"], softmax_scale=SCALE, **scales(c))
    few = {n: alone(x, n) for n in (0, N // 2 + 1, N - 1)}
    close = lambda a, b: bool(((a.float() - b.float()).abs() <= (2 * 2.0 ** -8 * b.float().abs() + 3e-3 if dtype == torch.bfloat16 else 2e-4)).all())
    o = tree(x, slice(None))
    for n, c in few.items():
        assert close(o[n:n + 1], tree(c, slice(n, n + 1))), n
    rb.rattn_tree_commit(k, v, parent, accepted, pos, x["kr"], x["vr"], x["state"], **scales(x))
    for n, c in few.items():
        i = slice(n, n + 1)
        rb.rattn_tree_commit(k[i], v[i], parent[i], accepted[i], pos[i], c["kr"], c["vr"], c["state"], **scales(c))
        assert same(alone(x, n), c), n
    if packed:
        step = lambda c, i: rb.rattn_decode_step_packed(q[i, 0].contiguous(), k[i, 1].contiguous(), v[i, 1].contiguous(), pos[i], c["kr"], c["ks"],
                                                        c["vr"], c["vs"], c["state"], softmax_scale=SCALE)
        o = step(x, slice(None))
        for n, c in few.items():
            assert close(o[n:n + 1], step(c, slice(n, n + 1))), n
            y = alone(x, n)
            assert same({t: y[t] for t in ("kr", "ks", "vr", "vs")}, {t: c[t] for t in ("kr", "ks", "vr", "vs")})
            assert float((y["state"] - c["state"]).abs().max()) <= 1e-5
        kr, vr = rb.rattn_ring_unpack(x["kr"], x["ks"], x["vr"], x["vs"])
        again = rb.rattn_ring_pack(kr, vr)
        for n in few:
            one = rb.rattn_ring_unpack(*(x[t][n:n + 1].contiguous() for t in ("kr", "ks", "vr", "vs")))
            assert torch.equal(kr[n:n + 1], one[0]) and torch.equal(vr[n:n + 1], one[1])
            assert torch.equal(rb.rattn_ring_unpack(*(t[n:n + 1].contiguous() for t in again))[0], one[0])


@pytest.mark.parametrize("packed", [False, True])
def test_one_ring(packed):
    """A ring of more than 2^32 bytes (8 bits: 2^31); keys that draw a row's attention lie at both ends and where offsets wrap."""
    D, W, G = 128, (1 << 24) + 37, 2
    x, r = cache(1, 1, W, D, torch.bfloat16, packed, 8960)
    p = 3 * W + 1000
    marks = [0, 999, 1000, 1001, (1 << 23) - 1, (1 << 23) + 1, 1 << 24, W - 1]     # (1000: the next slot)
    q, k, v = r(1, 1, G, D), r(1, 1, 1, D), r(1, 1, 1, D)
    at = torch.tensor(marks, device="cuda")
    mk = (30.0 * q[0, 0, :1].float() / q[0, 0, 0].float().norm()).bfloat16().repeat(len(marks), 1)[None, None]
    mv = r(1, 1, len(marks), D)
    if packed:
        codes = rb.rattn_ring_pack(mk.contiguous(), mv)
        for name, t in zip(("kr", "ks", "vr", "vs"), codes):
            x[name].view(torch.uint8)[0, 0, at] = t.view(torch.uint8)[0, 0]
        values = lambda a, b, i: (x[a][0, 0, i].double().view(-1, 4, 32) * x[b][0, 0, i].double()[..., None]).reshape(-1, D)
        row = lambda n, i: values("kr", "ks", i) if n == "k" else values("vr", "vs", i)
    else:
        x["kr"][0, 0, at], x["vr"][0, 0, at] = mk[0, 0], mv[0, 0]
        row = lambda n, i: x["kr" if n == "k" else "vr"][0, 0, i].double()
    # the formula in fp64: the node sees all ring tokens but the oldest, in slot 1000, and itself
    qd, slot = q[0, 0].double(), p % W
    num, den, top = torch.zeros(G, D, dtype=torch.float64, device="cuda"), torch.zeros(G, 1, dtype=torch.float64, device="cuda"), 60.0
    for a in range(0, W, 1 << 20):
        i = slice(a, min(a + (1 << 20), W))
        w = torch.exp(qd @ row("k", i).T * SCALE - top)
        if i.start <= slot < i.stop:
            w[:, slot - i.start] = 0.0
        num += w @ row("v", i)
        den += w.sum(1, keepdim=True)
    w = torch.exp((qd @ k[0, 0].double().T) * SCALE - top)
    num, den = num + w @ v[0, 0].double(), den + w
    gone = slice(slot, slot + 1)
    phi = lambda t: torch.softmax(t, -1)
    S = x["state"][0, 0].double() + phi(row("k", gone)).T @ row("v", gone)
    norm = lambda t: t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS)
    want = norm(num / den) + norm(phi(qd) @ S)
    pos = torch.tensor([p], dtype=torch.int32, device="cuda")
    parent = torch.tensor([[-1]], dtype=torch.int32, device="cuda")
    o = rb.rattn_tree_step(q, k, v, parent, pos, x["kr"], x["vr"], x["state"], softmax_scale=SCALE, k_scale=x.get("ks"), v_scale=x.get("vs"))
    bar = 2.0 ** -8 * want.abs() + 2e-2
    print(f"tree {float((o[0, 0].double() - want).abs().max()):.2e}", flush=True)
    assert bool(((o[0, 0].double() - want).abs() <= bar).all())
    if packed:
        o = rb.rattn_decode_step_packed(q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous(), pos, x["kr"], x["ks"], x["vr"], x["vs"],
                                        x["state"], softmax_scale=SCALE)
        assert bool(((o[0].double() - want).abs() <= bar).all())
        new = rb.rattn_ring_pack(k, v)
        assert torch.equal(x["kr"].view(torch.uint8)[0, 0, slot], new[0].view(torch.uint8)[0, 0, 0])
    else:
        rb.rattn_tree_commit(k, v, parent, torch.zeros(1, dtype=torch.int32, device="cuda"), pos, x["kr"], x["vr"], x["state"])
        assert torch.equal(x["kr"][0, 0, slot], k[0, 0, 0]) and torch.equal(x["vr"][0, 0, slot], v[0, 0, 0])
    assert float((x["state"][0, 0].double() - S).abs().max()) <= 1e-5 * max(1.0, float(S.abs().max()))
