"""Pins of the oracle's packed rings and trees of drafted tokens: brute force over the 8-bit numbers, and the layer's forward and
decode step on every path of a tree.  CPU only."""
import numpy as np
import pytest

from oracle import rattn_oracle as orc


def e4m3_numbers():
    """All finite E4M3 numbers that are not negative: codes 0 .. 126."""
    return np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).view(np.float32).astype(np.float64)


def test_codes_are_the_nearest_numbers_ties_to_even():
    num = e4m3_numbers()
    assert num[-1] == 448.0 and num[8] == 2.0 ** -6
    rng = np.random.default_rng(1)
    mid = (num[1:] + num[:-1]) / 2
    x = np.concatenate([num, mid, mid * (1 + 1e-7), mid * (1 - 1e-7), rng.uniform(0, 448, 4000), np.exp(rng.uniform(-9, 6, 4000))])
    x = np.concatenate([x, np.full(-len(x) % 31, 1.0)]).reshape(-1, 31)
    x = np.concatenate([x, np.full((len(x), 1), 448.0)], 1)          # the factor is 1
    codes, scales = orc.pack_rows(x)
    assert np.all(scales == 1.0)
    i = np.clip(np.searchsorted(num, x), 1, len(num) - 1)
    lo, hi = num[i - 1], num[i]
    near = np.where(x - lo < hi - x, lo, np.where(x - lo > hi - x, hi, np.where((i - 1) % 2 == 0, lo, hi)))
    assert np.array_equal(codes, near)


def test_factor_and_error_bounds():
    rng = np.random.default_rng(2)
    x = bf16(rng.standard_normal((300, 128)) * np.exp(rng.uniform(-40, 40, (300, 1))))
    codes, scales = orc.pack_rows(x)
    y = orc.packed_values(codes, scales)
    blocks = np.abs(x).reshape(300, 4, 32).max(-1)
    assert np.all(blocks <= 448 * scales) and np.all((blocks > 224 * scales) | (scales == 2.0 ** -126))
    assert np.all(np.abs(y - x) <= np.maximum(np.abs(x) / 16, np.repeat(scales, 32, -1) / 1024))
    again = orc.packed_values(*orc.pack_rows(y))
    assert np.array_equal(again, y)
    assert np.array_equal(bf16(y), y)                                  # bf16 holds what is stored
    special = np.zeros((1, 64)); special[0, 3] = np.inf; special[0, 4] = 2.0; special[0, 40] = np.nan
    codes, scales = orc.pack_rows(special)
    assert np.isnan(codes[0, [3, 40]]).all() and np.isfinite(np.delete(codes[0], [3, 40])).all()
    assert codes[0, 4] * scales[0, 0] == 2.0 and scales[0, 1] == 2.0 ** -126


def cache_after(k, v, W, fm):
    return orc.prefill_export(k, v, W, fm)


@pytest.mark.parametrize("fm", ["softmax", "relu"])
@pytest.mark.parametrize("p,W", [(0, 3), (2, 5), (5, 5), (6, 5), (20, 5), (9, 1), (9, 40)])
def test_tree_is_the_layer_on_every_path(p, W, fm):
    rng = np.random.default_rng(3 + p + W)
    M, Hq, Hkv, D = 7, 4, 2, 8
    parent = np.array([[-1, 0, 0, 1, -1, 3, 5]])
    q = rng.standard_normal((1, M, Hq, D)); k = rng.standard_normal((1, M, Hkv, D)); v = rng.standard_normal((1, M, Hkv, D))
    pk = rng.standard_normal((1, p, Hkv, D)); pv = rng.standard_normal((1, p, Hkv, D))
    kr, vr, S = cache_after(pk, pv, W, fm)
    o = orc.tree_step(q, k, v, parent, [p], kr, vr, S, W, scale=0.4, feature_map=fm)
    for i in range(M):
        path = orc.tree_path(parent[0], i)
        T = p + len(path)
        fq = np.zeros((1, T, Hq, D)); fq[:, p:] = q[:, path]
        fk = np.concatenate([pk, k[:, path]], 1); fv = np.concatenate([pv, v[:, path]], 1)
        want = orc.fwd_dense(fq, fk, fv, W, scale=0.4, feature_map=fm)["o"][0, -1]
        np.testing.assert_allclose(o[0, i], want, atol=1e-12)
        # accepting it leaves what a prompt of those tokens leaves (slots that no token reached apart)
        got = orc.tree_commit(k, v, parent, [i], [p], kr, vr, S, W, fm)
        for x, y in zip(got, cache_after(fk, fv, W, fm)):
            np.testing.assert_allclose(x, y, atol=1e-12)
    assert orc.tree_path([-1, 5, 1, -7], 2) == [1, 2] and orc.tree_path([-1, 0, 1, -7], 3) == [3]


def test_one_node_is_a_decode_step():
    rng = np.random.default_rng(5)
    N, Hq, Hkv, D, W = 3, 4, 1, 8, 4
    pos = [0, 4, 11]
    kr, vr = rng.standard_normal((2, N, Hkv, W, D)); S = rng.standard_normal((N, Hkv, D, D))
    S[:2] = 0
    q = rng.standard_normal((N, Hq, D)); k, v = rng.standard_normal((2, N, Hkv, D))
    o, kr2, vr2, S2 = orc.decode_step(q, k, v, pos, kr, vr, S, W, scale=0.3)
    parent = np.full((N, 1), -1)
    t = orc.tree_step(q[:, None], k[:, None], v[:, None], parent, pos, kr, vr, S, W, scale=0.3)
    np.testing.assert_allclose(t[:, 0], o, atol=1e-13)
    for x, y in zip(orc.tree_commit(k[:, None], v[:, None], parent, [0] * N, pos, kr, vr, S, W), (kr2, vr2, S2)):
        np.testing.assert_allclose(x, y, atol=1e-13)
