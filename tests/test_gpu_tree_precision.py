"""What a tree step's bf16 output is off by is its own rounding, whichever kernel the plan takes: a sequence is verified as well in a
large batch as in a small one."""
import numpy as np
import pytest
import torch

from test_gpu_tree import make, np64, oracle, step
from test_gpu_tree_tiles import kernels, some

pytestmark = pytest.mark.gpu


def norm(x):
    return float(np.sqrt((x * x).sum()))


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("N,M,Hq,Hkv,W,pos,tiles", [
    (260, 17, 8, 2, 300, 900, True), (70, 40, 32, 8, 150, 700, True), (520, 64, 2, 1, 33, 200, True),
    (3, 17, 8, 2, 300, 900, False), (2, 40, 32, 8, 150, 700, False), (1, 12, 16, 4, 2048, 5000, False)])
def test_the_output_is_off_by_its_own_rounding(N, M, Hq, Hkv, W, pos, tiles, D, packed):
    """With r the rounding of the output to bf16 (some 1.7e-3 of its norm) and e what the kernels' two-term operands leave: a term
    holds 8 bits, so two leave 2^-17 of a probability and 2^-16 of a feature product, a state entry's product or a weight, each in at
    most three products in a row: e <= 2^-14 of the norm, and sqrt(r^2 + e^2) <= 1.001 r.  One term for the probabilities (2^-9 of
    each at most, 1.3e-3 of the norm on average) makes it 1.28 r."""
    print(f"N={N} M={M} Hq={Hq} Hkv={Hkv} D={D} W={W} packed={packed}", flush=True)
    x = make(N, M, Hq, Hkv, D, W, "bf16", [pos + i for i in range(N)], packed, 8700 + M, 2)
    scale = D ** -0.5
    o = step(x, scale)
    assert kernels(lambda: step(x, scale)) == {"tree_tile_kernel" if tiles else "tree_kernel"}
    ns = sorted({0, N // 2, N - 1})
    ref = oracle(some(x, ns), W, scale)
    rounded = np64(torch.from_numpy(ref).to(torch.bfloat16))
    own, least = norm(np64(o[ns]) - ref), norm(rounded - ref)
    print(f"off by {own / norm(ref):.4e} of its norm, rounding alone {least / norm(ref):.4e}", flush=True)
    assert own <= 1.01 * least
