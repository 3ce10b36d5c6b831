"""Tree steps read no more of their inputs than belongs to them: whatever lies behind the last ring row and the last drafted token, in
memory or in the tensors themselves, changes no bit of a result (rows that meet something that is no number are formed again, in another
order, which gives other bits)."""
import pytest
import torch

from paper_2506_15545_amd import binding as rb
from test_gpu_tree import make, step

pytestmark = pytest.mark.gpu
BEHIND = 64 * 4 * 128 * 4     # bytes: more rows of keys than a set has


def with_something_behind(t, byte):
    """A copy of t at the start of an allocation that goes on with `byte`s (0xFF: NaN in every type here)."""
    n = t.numel() * t.element_size()
    full = torch.full((n + BEHIND,), byte, dtype=torch.uint8, device="cuda")
    view = full[:n].view(t.dtype).view(t.shape)
    view.view(torch.uint8).copy_(t.contiguous().view(torch.uint8))
    return view


def both(x, scale, **kw):
    """The step's results with zeros and with NaN behind the keys and values."""
    got = []
    for byte in (0, 0xFF):
        y = dict(x)
        for n in ("k", "v", "kr", "vr", "ks", "vs"):
            if x[n] is not None:
                y[n] = with_something_behind(x[n], byte)
        got.append(step(y, scale, **kw))
    return got


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("M,pos,W,G", [(1, 1, 300, 4), (5, 5, 300, 4), (17, 17, 300, 4), (1, 400, 17, 2), (5, 400, 1, 3), (17, 40, 5, 1),
                                       (3, 2100, 2049, 4), (33, 500, 100, 8), (40, 0, 9, 5)])
def test_what_lies_behind_the_tensors(M, pos, W, G, dtype, D, packed):
    print(f"M={M} pos={pos} W={W} G={G} {dtype} D={D} packed={packed}", flush=True)
    x = make(1, M, 2 * G, 2, D, W, dtype, [pos], packed, 8400 + M + W, 2)
    zero, nan = both(x, D ** -0.5)
    assert bool(torch.isfinite(zero).all()) and torch.equal(zero, nan)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count", [1, 5, 17])
def test_drafted_tokens_behind_the_count_and_slots_without_a_token(count, dtype, packed):
    M, W, D = 40, 90, 128
    x = make(2, M, 8, 2, D, W, dtype, [200, 33], packed, 8500 + count, 2)
    n = torch.tensor([count, count], dtype=torch.int32, device="cuda")
    want = step(x, 0.1, count=n)
    for name in ("q", "k", "v"):
        x[name][:, count:] = float("nan")
    for name in ("kr", "vr") + (("ks", "vs") if packed else ()):
        x[name].view(torch.uint8)[1, :, 33:] = 0xFF
    for got in both(x, 0.1, count=n):
        assert torch.equal(got, want)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_many_rows(D, packed):
    N, M, W = 260, 17, 45
    x = make(N, M, 8, 2, D, W, "bf16", [(33, 200)[i % 2] for i in range(N)], packed, 8600, 2)
    zero, nan = both(x, 0.1)
    assert bool(torch.isfinite(zero).all()) and torch.equal(zero, nan)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("N,M", [(3, 6), (260, 17)])
@pytest.mark.parametrize("counts", [True, False])
def test_sequences_without_work_are_zero_in_a_new_output(counts, N, M, native, monkeypatch):
    """Whatever the memory held that the output is made of: a sequence with pos < 0 is zero, as are the rows behind a count."""
    if not native:
        monkeypatch.setattr(rb._native, "tree_step", rb._no_native, raising=False)
    x = make(N, M, 8, 2, 128, 40, "bf16", [(70, -1, 20)[i % 3] for i in range(N)], False, 8700, 2)
    count = torch.full((N,), M - 2, dtype=torch.int32, device="cuda") if counts else None
    idle = torch.arange(N) % 3 == 1
    torch.cuda.synchronize()
    for _ in range(3):
        left = torch.full_like(x["q"], float("nan"))     # goes back to the allocator, which hands it out next
        del left
        o = step(x, 0.1, count=count)
        assert bool((o[idle] == 0).all()) and bool(torch.isfinite(o).all()) and bool((o[~idle][:, : M - 2] != 0).any())
        if counts:
            assert bool((o[:, M - 2:] == 0).all())
