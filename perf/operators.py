"""Operators over the layer's cache (a W-slot ring of keys and values and one D x D state per KV head), as a serving program
runs them: rings in 8 bits, and drafted tokens that are verified before they become part of the cache.

A case is a dict of plain values; `kind` names the operator:

  pack     rattn_ring_pack: rings in the tensors' type become rings in 8 bits
  unpack   rattn_ring_unpack: the way back
  decode   rattn_decode_step_packed: one new token for each of N sequences over rings in 8 bits
  tree     rattn_tree_step: the layer for a tree of M drafted tokens behind each of N sequences; the cache is read only
  commit   rattn_tree_commit: the accepted path of such a tree enters the cache

Rings in 8 bits: every 32 features of a row share a power of two (E8M0), the least one with which the largest finite of them is
at most 448, and are held as E4M3 numbers times it; what is no finite number is held as NaN.

`own` false: the plain form of each operator in elementary tensor operations; true: the library's.
"""
import math

import torch

own = False
EPS = 1e-6
MAXNODES = 64
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ring(name, kind, N, Hkv, D, W, dtype="bf16"):
    return dict(name=name, kind=kind, N=N, Hkv=Hkv, D=D, W=W, dtype=dtype)


def _decode(name, N, Hq, Hkv, D, W, pos_lo, pos_hi, dtype="bf16", gains=True):
    return dict(name=name, kind="decode", N=N, Hq=Hq, Hkv=Hkv, D=D, W=W, pos_lo=pos_lo, pos_hi=pos_hi, dtype=dtype, gains=gains)


def _tree(name, kind, N, Hq, Hkv, D, W, M, spread, pos_lo, pos_hi, packed, dtype="bf16", gains=True):
    # spread: a node's parent is one of the `spread` nodes before it (1: a chain)
    return dict(name=name, kind=kind, N=N, Hq=Hq, Hkv=Hkv, D=D, W=W, M=M, spread=spread, pos_lo=pos_lo, pos_hi=pos_hi,
                packed=packed, dtype=dtype, gains=gains)


def listed():
    return [
        # one conversation's rings after its prompt (4 KV heads, window 512)
        _ring("pack_one", "pack", 1, 4, 128, 512),
        # the rings of the decode benchmark's batch
        _ring("pack_batch", "pack", 128, 8, 128, 512),
        # a few small-headed fp32 sequences of odd window, read back to continue a prompt
        _ring("unpack_ragged", "unpack", 3, 8, 64, 589, dtype="f32"),
        # a moderate batch with a wide window, read back
        _ring("unpack_wide", "unpack", 24, 8, 128, 2048),
        # one sequence being generated interactively
        _decode("decode_one", 1, 16, 4, 128, 512, 2000, 2000),
        # batch serving: the decode benchmark's step
        _decode("decode_batch", 128, 32, 8, 128, 512, 512, 32768, gains=False),
        # a moderate batch on the 12B layer (40 query / 8 KV heads) with a wider window, half of the sequences still inside it
        _decode("decode_wide", 24, 40, 8, 128, 2048, 100, 4000),
        # one conversation with a small tree of drafts
        _tree("tree_one", "tree", 1, 16, 4, 128, 512, 12, 3, 2000, 2000, False),
        # batch serving with short chains of drafts, rings in 8 bits
        _tree("tree_batch", "tree", 64, 32, 8, 128, 512, 6, 1, 300, 32768, True),
        # large trees on the 12B layer with a wide window, half of the sequences still inside it
        _tree("tree_large", "tree", 24, 40, 8, 128, 2048, 61, 8, 100, 4000, False),
        # the accepted tokens of one conversation
        _tree("commit_one", "commit", 1, 16, 4, 128, 512, 12, 3, 2000, 2000, False),
        # those of the decode benchmark's batch, rings in 8 bits
        _tree("commit_batch", "commit", 128, 32, 8, 128, 512, 6, 1, 512, 32768, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pack", "unpack", "decode", "decode", "tree", "tree", "tree", "commit"])
    Hkv, G = rng.choice([(8, 1), (8, 4), (8, 5), (4, 4), (4, 2), (2, 8), (2, 1), (1, 20)])
    D, W = rng.choice([128, 128, 128, 64]), _log_int(rng, 16, 4096)
    if rng.random() < 0.4:   # aligned windows are as common as odd ones
        W = (W + 63) // 64 * 64
    dtype = rng.choice(["bf16"] * 4 + ["f32"])
    N = max(1, min(_log_int(rng, 1, 128), int(6.7e7 / (W * Hkv * D))))
    if kind in ("pack", "unpack"):
        return dict(kind=kind, N=N, Hkv=Hkv, D=D, W=W, dtype=dtype)
    hi = _log_int(rng, 16, 32768)
    lo, gains = rng.randrange(0, hi), rng.random() < 0.6
    if kind == "decode":
        return dict(kind="decode", N=N, Hq=Hkv * G, Hkv=Hkv, D=D, W=W, pos_lo=lo, pos_hi=hi, dtype=dtype, gains=gains)
    M, spread = _log_int(rng, 1, MAXNODES), rng.choice([1, 1, 2, 4, 8])
    case = dict(kind=kind, N=N, Hq=Hkv * G, Hkv=Hkv, D=D, W=W, M=M, spread=spread, pos_lo=lo, pos_hi=hi,
                packed=rng.random() < 0.5, dtype=dtype, gains=gains)
    while kind == "tree" and work(case)["flops"] > (6e10 if dtype == "bf16" else 6e9):
        if case["N"] > 1:
            case["N"] //= 2
        else:
            case["M"] = max(1, case["M"] // 2)
            if case["M"] == 1:
                break
    return case


def _scale(D):
    return 1.0 / math.sqrt(D)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = _TYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)

    N, Hkv, D, W = case["N"], case["Hkv"], case["D"], case["W"]
    s = {"case": case, "gs": None, "gr": None, "ks": None, "vs": None}
    packed = case["kind"] in ("unpack", "decode") or case.get("packed", False)
    s["kr"], s["vr"] = normal(N, Hkv, W, D), normal(N, Hkv, W, D)
    if packed:
        (s["kr"], s["ks"]), (s["vr"], s["vs"]) = _pack(s["kr"]), _pack(s["vr"])
    if case["kind"] == "pack":
        s["out"] = tuple(torch.zeros(N, Hkv, W, n, dtype=torch.uint8, device="cuda").view(t)
                         for n, t in ((D, torch.float8_e4m3fn), (D // 32, torch.float8_e8m0fnu)) * 2)
        return s
    if case["kind"] == "unpack":
        s["out"] = tuple(torch.zeros(N, Hkv, W, D, dtype=dt, device="cuda") for _ in range(2))
        return s
    Hq = case["Hq"]
    if case["gains"] and case["kind"] != "commit":
        s["gs"], s["gr"] = (1.0 + 0.1 * normal(Hq, D, dtype=torch.float32) for _ in range(2))
    s["pos"] = torch.randint(case["pos_lo"], case["pos_hi"] + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
    # a sum of pos - W outer products of a softmax row of a normal key with a normal value
    std = torch.sqrt(torch.clamp(s["pos"].float() - W, min=0.0) * math.e) / D
    s["state"] = normal(N, Hkv, D, D, dtype=torch.float32) * std.view(N, 1, 1, 1)
    if case["kind"] == "decode":
        s["q"], s["k"], s["v"] = normal(N, Hq, D), normal(N, Hkv, D), normal(N, Hkv, D)
        s["o"] = torch.zeros_like(s["q"])
        return s
    M = case["M"]
    s["k"], s["v"] = normal(N, M, Hkv, D), normal(N, M, Hkv, D)
    back = torch.randint(0, case["spread"], (N, M), generator=g, device="cuda", dtype=torch.int32)
    s["parent"] = torch.clamp(torch.arange(M, device="cuda", dtype=torch.int32) - 1 - back, min=-1).contiguous()
    s["count"] = torch.randint((M + 1) // 2, M + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
    if case["kind"] == "tree":
        s["q"] = normal(N, M, Hq, D)
        s["o"] = torch.zeros_like(s["q"])
    else:
        part = torch.rand(N, generator=g, device="cuda")
        s["accepted"] = (torch.floor(part * (s["count"] + 1).float()) - 1).to(torch.int32)
    return s


# ------------------------------------------------------------------ plain forms
def _pack(x):
    """Codes and scales of rows [..., D]."""
    y = x.float().unflatten(-1, (-1, 32))
    a = torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y)).amax(-1)
    m, ex = torch.frexp(a)                                        # a = m 2^ex, 448 = 0.875 * 2^9
    e = torch.where(a > 0, torch.clamp(ex - 9 + (m > 0.875).int(), min=-126), torch.full_like(ex, -126))
    codes = y * ((127 - e) << 23).view(torch.float32)[..., None]       # 2^-e, to the bit
    return codes.flatten(-2).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _unpack(codes, scale):
    return (codes.float().unflatten(-1, (-1, 32)) * scale.float()[..., None]).flatten(-2)


def _phi(x):
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _rms(x, gain):
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return y if gain is None else y * gain


def _softmax(a):
    e = torch.exp(a - a.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _rings(s):
    if s["ks"] is None:
        return s["kr"].float(), s["vr"].float()
    return _unpack(s["kr"], s["ks"]), _unpack(s["vr"], s["vs"])


def _into(ring, rows, where):
    """`rows` (or bytes of them) into the places of `ring` that `where` marks, in place."""
    bits = torch.uint8 if ring.element_size() == 1 else ring.dtype
    r = ring.view(bits)
    r.copy_(torch.where(where, rows.view(bits), r))


def _ages(s):
    """Of every slot: the age index j of its token (0: the oldest of a full ring), and whether it holds one."""
    W, pos = s["case"]["W"], s["pos"].long()[:, None]
    slot, first = torch.arange(W, device="cuda")[None], pos % W
    j = slot - first + torch.where(slot < first, W, 0)
    return j, j >= W - pos


def _closure(s):
    """[N,M,M]: whether column j is row i or one of its ancestors; and every node's depth."""
    M = s["case"]["M"]
    up = (s["parent"].long()[..., None] == torch.arange(M, device="cuda")).float()
    anc = torch.linalg.matrix_power(torch.eye(M, device="cuda") + up, M) > 0
    return anc, anc.sum(-1) - 1


def _plain_decode(s):
    case = s["case"]
    N, Hq, Hkv, D, W = (case[n] for n in ("N", "Hq", "Hkv", "D", "W"))
    pos = s["pos"].long()
    q, kn, vn = s["q"].float().view(N, Hkv, Hq // Hkv, D), s["k"].float(), s["v"].float()
    K, V = _rings(s)
    slots = torch.arange(W, device="cuda")[None]
    new = slots == (pos % W)[:, None]                                       # [N,W]
    at = new[:, None, :, None]
    old_k, old_v = (K * at).sum(2), (V * at).sum(2)
    evict = (pos >= W)[:, None, None, None]
    s["state"].copy_(torch.where(evict, s["state"] + _phi(old_k)[..., None] * old_v[..., None, :], s["state"]))
    K, V = torch.where(at, kn[:, :, None], K), torch.where(at, vn[:, :, None], V)
    see = slots < torch.clamp(pos + 1, max=W)[:, None]
    a = torch.matmul(q, K.transpose(-1, -2)) * _scale(D)
    xs = torch.matmul(_softmax(torch.where(see[:, None, None], a, torch.full_like(a, -math.inf))), V)
    xr = torch.matmul(_phi(q), s["state"])
    gs, gr = ((None, None) if s["gs"] is None else (g.view(Hkv, Hq // Hkv, D) for g in (s["gs"], s["gr"])))
    s["o"].copy_((_rms(xs, gs) + _rms(xr, gr)).view(N, Hq, D))
    (kc, ks), (vc, vs) = _pack(kn), _pack(vn)
    _into(s["kr"], kc.view(torch.uint8)[:, :, None], at)
    _into(s["vr"], vc.view(torch.uint8)[:, :, None], at)
    _into(s["ks"], ks.view(torch.uint8)[:, :, None], at)
    _into(s["vs"], vs.view(torch.uint8)[:, :, None], at)
    return s["o"]


def _plain_tree(s):
    case = s["case"]
    N, Hq, Hkv, D, W, M = (case[n] for n in ("N", "Hq", "Hkv", "D", "W", "M"))
    G = Hq // Hkv
    K, V = _rings(s)
    K, V = torch.cat([K, s["k"].float().transpose(1, 2)], 2), torch.cat([V, s["v"].float().transpose(1, 2)], 2)
    anc, depth = _closure(s)
    j, there = _ages(s)
    inside = torch.cat([there[:, None] & (j[:, None] > depth[..., None]), anc & (depth[..., None] - depth[:, None] < W)], -1)
    left = torch.cat([there[:, None] & (j[:, None] <= depth[..., None]), anc & (depth[..., None] - depth[:, None] >= W)], -1)
    q = s["q"].float().view(N, M, Hkv, G, D).permute(0, 2, 1, 3, 4)         # [N,Hkv,M,G,D]
    a = torch.matmul(q.reshape(N, Hkv, M * G, D), K.transpose(-1, -2)).view(N, Hkv, M, G, W + M) * _scale(D)
    p = _softmax(torch.where(inside[:, None, :, None], a, torch.full_like(a, -math.inf)))
    xs = torch.matmul(p.view(N, Hkv, M * G, W + M), V)
    fq = _phi(q).reshape(N, Hkv, M * G, D)
    c = torch.matmul(fq, _phi(K).transpose(-1, -2)).view(N, Hkv, M, G, W + M) * left[:, None, :, None]
    S = torch.where((s["pos"] > W)[:, None, None, None], s["state"], torch.zeros_like(s["state"]))
    xr = torch.matmul(c.view(N, Hkv, M * G, W + M), V) + torch.matmul(fq, S)
    gs, gr = ((None, None) if s["gs"] is None else (g.view(Hkv, 1, G, D) for g in (s["gs"], s["gr"])))
    o = _rms(xs.view(N, Hkv, M, G, D), gs) + _rms(xr.view(N, Hkv, M, G, D), gr)
    o = o.permute(0, 2, 1, 3, 4).reshape(N, M, Hq, D).to(s["o"].dtype)
    row = torch.arange(M, device="cuda")[None] < s["count"][:, None]
    s["o"].copy_(torch.where(row[..., None, None], o, s["o"]))
    return s["o"]


def _plain_commit(s):
    case = s["case"]
    N, Hkv, D, W, M = (case[n] for n in ("N", "Hkv", "D", "W", "M"))
    pos, acc = s["pos"].long(), s["accepted"].long()
    K, V = _rings(s)
    kn, vn = s["k"].transpose(1, 2), s["v"].transpose(1, 2)                 # [N,Hkv,M,D]
    K, V = torch.cat([K, kn.float()], 2), torch.cat([V, vn.float()], 2)
    anc, depth = _closure(s)
    mine = torch.gather(anc, 1, torch.clamp(acc, min=0)[:, None, None].expand(N, 1, M))[:, 0] & (acc >= 0)[:, None]   # [N,M]
    n = mine.sum(-1, keepdim=True)
    j, there = _ages(s)
    leave = torch.cat([there & (j < n), mine & (depth < n - W)], -1)[:, None, :, None]
    S = torch.where((pos > W)[:, None, None, None], s["state"], torch.zeros_like(s["state"]))
    folded = S + torch.matmul((_phi(K) * leave).transpose(-1, -2), V)
    s["state"].copy_(torch.where(leave.any(2, keepdim=True), folded, s["state"]))
    # [N,W,M]: the path's node that a slot receives
    to = mine[:, None] & (depth >= n - W)[:, None] & \
        ((pos[:, None] + depth) % W)[:, None].eq(torch.arange(W, device="cuda")[None, :, None])
    at, node = to.any(-1)[:, None, :, None], to.int().argmax(-1)

    def place(ring, rows):   # rows [N,Hkv,M,n]
        rows = rows.view(torch.uint8) if rows.element_size() == 1 else rows
        index = node[:, None, :, None].expand(N, Hkv, W, rows.shape[-1])
        _into(ring, torch.gather(rows, 2, index), at)

    if s["ks"] is None:
        place(s["kr"], kn)
        place(s["vr"], vn)
    else:
        (kc, ks), (vc, vs) = _pack(kn), _pack(vn)
        place(s["kr"], kc)
        place(s["vr"], vc)
        place(s["ks"], ks)
        place(s["vs"], vs)


def run(s):
    case = s["case"]
    kind, dt = case["kind"], _TYPES[case["dtype"]]
    cache = {"kr": s["kr"], "vr": s["vr"], "ks": s["ks"], "vs": s["vs"], "state": s.get("state")}
    if own:
        from paper_2506_15545_amd import binding as rb

    if kind == "pack":
        if own:
            return rb.rattn_ring_pack(s["kr"], s["vr"], out=s["out"])
        for t, x in zip(s["out"], _pack(s["kr"]) + _pack(s["vr"])):
            t.copy_(x)
        return s["out"]
    if kind == "unpack":
        if own:
            return rb.rattn_ring_unpack(s["kr"], s["ks"], s["vr"], s["vs"], dt, out=s["out"])
        s["out"][0].copy_(_unpack(s["kr"], s["ks"]))
        s["out"][1].copy_(_unpack(s["vr"], s["vs"]))
        return s["out"]
    if kind == "decode":
        if own:
            rb.rattn_decode_step_packed(s["q"], s["k"], s["v"], s["pos"], s["kr"], s["ks"], s["vr"], s["vs"], s["state"],
                                        s["gs"], s["gr"], softmax_scale=_scale(case["D"]), out=s["o"])
        else:
            _plain_decode(s)
        return {"o": s["o"], **cache}
    if kind == "tree":
        if own:
            return rb.rattn_tree_step(s["q"], s["k"], s["v"], s["parent"], s["pos"], s["kr"], s["vr"], s["state"], s["gs"],
                                      s["gr"], softmax_scale=_scale(case["D"]), count=s["count"], k_scale=s["ks"],
                                      v_scale=s["vs"], out=s["o"])
        return _plain_tree(s)
    if own:
        rb.rattn_tree_commit(s["k"], s["v"], s["parent"], s["accepted"], s["pos"], s["kr"], s["vr"], s["state"],
                             k_scale=s["ks"], v_scale=s["vs"])
    else:
        _plain_commit(s)
    return cache


# ------------------------------------------------------------------ what a pass cannot do without
def _mean_min(lo, hi, cap):
    """Mean of min(p, cap) over p = lo .. hi, and the share of p >= cap."""
    n, k = hi - lo + 1, max(0, min(hi, cap - 1) - lo + 1)
    return (k * (2 * lo + k - 1) / 2 + (n - k) * cap) / n, (n - k) / n


def work(case):
    N, Hkv, D, W = case["N"], case["Hkv"], case["D"], case["W"]
    e, row8 = (4 if case["dtype"] == "f32" else 2), D + D // 32
    if case["kind"] in ("pack", "unpack"):
        return {"bytes": 2 * N * Hkv * W * (D * e + row8), "flops": 2 * N * Hkv * W * D}
    Hq = case["Hq"]
    rows, full = _mean_min(case["pos_lo"], case["pos_hi"], W)
    if case["kind"] == "decode":
        nbytes = N * (2 * Hkv * (rows * row8 + D * D * 4 * full) + (2 * Hq + 2 * Hkv) * D * e + 2 * Hkv * row8)
        return {"bytes": nbytes, "flops": N * (4 * Hq * D * (rows + 1) + (2 * Hq + 2 * Hkv * full) * D * D)}
    # nodes of a sequence, and the mean length of a path through them
    M = (case["M"] + (case["M"] + 1) // 2) / 2
    path = max(1.0, 1 + (M - 1) / 2 * 2 / (case["spread"] + 1))
    ring_row = row8 if case["packed"] else D * e
    if case["kind"] == "tree":
        flops = N * M * Hq * (4 * D * (rows + path) + 2 * D * D * full)
        return {"bytes": N * (2 * Hkv * rows * ring_row + Hkv * D * D * 4 * full + M * (2 * Hq + 2 * Hkv) * D * e), "flops": flops}
    half = path * M / (M + 1)    # one of the M + 1 outcomes accepts nothing
    nbytes = N * Hkv * full * (2 * D * D * 4 + 2 * half * ring_row) + N * Hkv * 2 * half * (D * e + ring_row)
    return {"bytes": nbytes, "flops": N * Hkv * full * half * 2 * D * D + 1}


# ------------------------------------------------------------------ from the definition, in 64 bits
def _values(codes, scale):
    c = codes.double()
    return c if scale is None else c * scale.double().repeat_interleave(32, -1)


def _two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)               # 2^e, to the bit


def _round8(x):
    """(values of the E4M3 codes, values of the scales) of rows [..., D] in 64 bits."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    a = b.masked_fill(~torch.isfinite(b), 0.0).abs().max(-1)[0]
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -150) / 448.0))
    e = torch.where(a > 448.0 * _two(e), e + 1, e)           # (the logarithm is rounded)
    e = torch.where(a <= 448.0 * _two(e - 1), e - 1, e).clamp(min=-126.0)
    y = b / _two(e)[..., None]
    step = _two(torch.floor(torch.log2(torch.nan_to_num(y, nan=1.0, posinf=1.0, neginf=1.0).abs().clamp(min=2.0 ** -6))) - 3)
    y = torch.where(torch.isfinite(y), torch.round(y / step) * step, torch.full_like(y, math.nan))
    return y.reshape(x.shape), _two(e)


def _feature(x):
    return torch.softmax(x, -1)


def _combine(xs, xr, gs, gr):
    n1 = xs / torch.sqrt((xs ** 2).mean(-1, keepdim=True) + EPS)
    n2 = xr / torch.sqrt((xr ** 2).mean(-1, keepdim=True) + EPS)
    return (n1 if gs is None else n1 * gs.double()) + (n2 if gr is None else n2 * gr.double())


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "pack":
        return _round8(s["kr"]) + _round8(s["vr"])
    if kind == "unpack":
        return _values(s["kr"], s["ks"]), _values(s["vr"], s["vs"])
    N, Hq, Hkv, D, W = (case[n] for n in ("N", "Hq", "Hkv", "D", "W"))
    G, state = Hq // Hkv, s["state"].double()
    # what run() returns of the rings: codes and scales apart, or the ring itself
    kr, vr = s["kr"].double(), s["vr"].double()
    ks, vs = (None, None) if s["ks"] is None else (s["ks"].double(), s["vs"].double())
    K, V = _values(s["kr"], s["ks"]), _values(s["vr"], s["vs"])

    def write(n, t, k, v):   # token t of sequence n, rows k, v [Hkv,D]
        if ks is None:
            kr[n, :, t % W], vr[n, :, t % W] = k, v
        else:
            (kr[n, :, t % W], ks[n, :, t % W]), (vr[n, :, t % W], vs[n, :, t % W]) = _round8(k), _round8(v)

    if kind == "decode":
        o = torch.zeros(N, Hq, D, dtype=torch.float64, device="cuda")
        for n, p in enumerate(s["pos"].tolist()):
            kn, vn = s["k"][n].double(), s["v"][n].double()
            tokens = torch.arange(max(0, p - W + 1), p, device="cuda") % W
            keys, vals = torch.cat([K[n][:, tokens], kn[:, None]], 1), torch.cat([V[n][:, tokens], vn[:, None]], 1)
            if p >= W:
                state[n] += _feature(K[n, :, p % W])[:, :, None] * V[n, :, p % W][:, None]
            q = s["q"][n].double().view(Hkv, G, D)
            xs = torch.softmax(q @ keys.mT / math.sqrt(D), -1) @ vals
            o[n] = _combine(xs.view(Hq, D), (_feature(q) @ state[n]).view(Hq, D), s["gs"], s["gr"])
            write(n, p, kn, vn)
        return {"o": o, "kr": kr, "vr": vr, "ks": ks, "vs": vs, "state": state}

    M, parents = case["M"], s["parent"].tolist()
    o = torch.zeros(N, M, Hq, D, dtype=torch.float64, device="cuda")
    for n, p in enumerate(s["pos"].tolist()):
        old = torch.arange(max(0, p - W), p, device="cuda") % W             # ring tokens in order
        nring = old.numel()
        keys = torch.cat([K[n][:, old], s["k"][n].double().transpose(0, 1)], 1)     # [Hkv, ring + M, D]
        vals = torch.cat([V[n][:, old], s["v"][n].double().transpose(0, 1)], 1)
        S = state[n] if p > W else torch.zeros_like(state[n])
        paths = []
        for i in range(M):
            up = parents[n][i]
            paths.append((paths[up] if up >= 0 else []) + [i])
        if kind == "commit":
            a = int(s["accepted"][n])
            path = paths[a] if a >= 0 else []
            line = list(range(nring)) + [nring + i for i in path]           # tokens p - nring ..., in order
            gone = line[:max(0, len(line) - W)]
            if gone:
                state[n] = S + _feature(keys[:, gone]).mT @ vals[:, gone]
            for d, i in enumerate(path):
                write(n, p + d, s["k"][n, i].double(), s["v"][n, i].double())
            continue
        nodes = int(s["count"][n])
        inside = torch.zeros(M, nring + M, dtype=torch.bool)
        left = torch.zeros(M, nring + M, dtype=torch.bool)
        for i in range(nodes):
            line = torch.tensor(list(range(nring)) + [nring + x for x in paths[i]])
            inside[i, line[max(0, len(line) - W):]] = True
            left[i, line[:max(0, len(line) - W)]] = True
        inside, left = inside.cuda(), left.cuda()
        q = s["q"][n].double().view(M, Hkv, G, D)[:nodes].transpose(0, 1)           # [Hkv,nodes,G,D]
        a = (q.reshape(Hkv, nodes * G, D) @ keys.mT).view(Hkv, nodes, G, -1) / math.sqrt(D)
        prob = torch.softmax(a.masked_fill(~inside[:nodes, None], -math.inf), -1)
        xs = prob.reshape(Hkv, nodes * G, -1) @ vals
        f = _feature(q).reshape(Hkv, nodes * G, D)
        c = (f @ _feature(keys).mT).view(Hkv, nodes, G, -1).masked_fill(~left[:nodes, None], 0.0)
        xr = c.reshape(Hkv, nodes * G, -1) @ vals + f @ S
        heads = [x.view(Hkv, nodes, G, D).transpose(0, 1).reshape(nodes, Hq, D) for x in (xs, xr)]
        o[n, :nodes] = _combine(*heads, s["gs"], s["gr"])
    return o if kind == "tree" else {"kr": kr, "vr": vr, "ks": ks, "vs": vs, "state": state}
