"""Packed rings and trees of drafted tokens: what the C ABI and the binding refuse, on the host, before anything is launched; and the
host layer under AddressSanitizer and UndefinedBehaviorSanitizer."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2506_15545_amd import binding as rb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(1 << 20)      # never dereferenced: the checks fail first
ODD = ctypes.c_void_p((1 << 20) + 8)


def decode_params(**kw):
    d = dict(N=2, Hq=4, Hkv=2, D=64, window=16, dtype=rb.RATTN_BF16, softmax_scale=1.0, rms_eps=1e-6, feature_map=0)
    return rb.RattnDecodeParams(**{**d, **kw})


def tree_params(**kw):
    d = dict(N=2, Hq=4, Hkv=2, D=64, window=16, dtype=rb.RATTN_BF16, nodes=5, softmax_scale=1.0, rms_eps=1e-6, feature_map=0)
    return rb.RattnTreeParams(**{**d, **kw})


BAD = [(dict(N=0), -1), (dict(Hq=3), -1), (dict(window=0), -1), (dict(rms_eps=0.0), -1), (dict(softmax_scale=0.0), -1),
       (dict(D=96), -2), (dict(dtype=2), -2), (dict(feature_map=3), -2), (dict(N=70000), -2), (dict(window=2 ** 31 - 1, N=60000), -2)]


@pytest.mark.parametrize("kw,code", BAD)
def test_bad_parameters(kw, code):
    L, n = rb.lib(), ctypes.c_size_t()
    p, t = decode_params(**kw), tree_params(**kw)
    assert L.rattn_decode_packed_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == code
    assert L.rattn_ring_pack(ctypes.byref(p), *[FAKE] * 6, None) == code
    assert L.rattn_ring_unpack(ctypes.byref(p), *[FAKE] * 6, None) == code
    assert L.rattn_decode_step_packed(ctypes.byref(p), *[FAKE] * 9, None, None, FAKE, None, 0, None) == code
    assert L.rattn_tree_workspace_bytes(ctypes.byref(t), 0, ctypes.byref(n)) == code
    assert L.rattn_tree_step(ctypes.byref(t), *[FAKE] * 11, None, None, FAKE, None, 0, None) == code
    assert L.rattn_tree_commit(ctypes.byref(t), *[FAKE] * 10, None) == code
    assert rb.lib().rattn_last_error()


def test_node_counts():
    L, n = rb.lib(), ctypes.c_size_t()
    for nodes, code in ((0, -1), (-3, -1), (65, -2), (1, 0), (64, 0)):
        assert L.rattn_tree_workspace_bytes(ctypes.byref(tree_params(nodes=nodes)), 0, ctypes.byref(n)) == code, nodes
    # rows of a node's tensors beyond 32-bit offsets, more work-groups than a launch has
    assert L.rattn_tree_workspace_bytes(ctypes.byref(tree_params(Hq=65536, Hkv=65536, nodes=64, D=128)), 0, ctypes.byref(n)) == -2
    assert L.rattn_tree_workspace_bytes(ctypes.byref(tree_params(N=65535, Hq=60000, Hkv=1, nodes=64)), 0, ctypes.byref(n)) == -2
    assert L.rattn_tree_workspace_bytes(None, 0, ctypes.byref(n)) == -1


def test_pointers_and_workspaces():
    L, n = rb.lib(), ctypes.c_size_t()
    p, t = decode_params(), tree_params()
    calls = {
        "rattn_ring_pack": (p, [FAKE] * 6, range(6), []),
        "rattn_ring_unpack": (p, [FAKE] * 6, range(6), []),
        "rattn_decode_step_packed": (p, [FAKE] * 9 + [None, None, FAKE, None, 0], [0, 1, 2, 3, 4, 5, 6, 7, 8, 11], [3]),
        # q k v parent count pos kr ks vr vs state gs gr o ws bytes
        "rattn_tree_step": (t, [FAKE] * 4 + [None] + [FAKE] * 6 + [None, None, FAKE, None, 0], [0, 1, 2, 3, 5, 6, 7, 8, 9, 10, 13], [3, 5]),
        "rattn_tree_commit": (t, [FAKE] * 10, range(10), [2, 3, 4]),
    }
    for name, (par, args, need, plain_ints) in calls.items():
        f = getattr(L, name)
        for i in need:
            a = list(args)
            a[i] = None
            assert f(ctypes.byref(par), *a, None) == -1, (name, i)
            if i not in plain_ints:      # (int32 arrays need no more than their own alignment)
                a[i] = ODD
                assert f(ctypes.byref(par), *a, None) == -1 and b"aligned" in L.rattn_last_error(), (name, i)
    # workspaces: reported, and refused when short
    p, t = decode_params(N=1, Hq=4, Hkv=1, D=128, window=4096), tree_params(N=1, Hq=4, Hkv=1, D=128, window=4096)
    assert L.rattn_decode_packed_workspace_bytes(ctypes.byref(p), ctypes.byref(n)) == 0 and n.value > 0
    st = L.rattn_decode_step_packed(ctypes.byref(p), *[FAKE] * 9, None, None, FAKE, FAKE, n.value - 1, None)
    assert st == -3 and b"workspace" in L.rattn_last_error()
    assert L.rattn_tree_workspace_bytes(ctypes.byref(t), 0, ctypes.byref(n)) == 0 and n.value > 0
    st = L.rattn_tree_step(ctypes.byref(t), *[FAKE] * 6, FAKE, None, FAKE, None, FAKE, None, None, FAKE, FAKE, n.value - 1, None)
    assert st == -3 and b"workspace" in L.rattn_last_error()
    # many sequences: nothing to share
    assert L.rattn_tree_workspace_bytes(ctypes.byref(tree_params(N=4096)), 1, ctypes.byref(n)) == 0 and n.value == 0


def tensors(N=2, M=3, Hq=4, Hkv=2, D=64, W=8, dtype=torch.bfloat16):
    z = lambda *s, dt=dtype: torch.zeros(*s, dtype=dt)
    codes = lambda n, dt: torch.zeros(N, Hkv, W, n, dtype=torch.uint8).view(dt)
    return dict(q=z(N, M, Hq, D), k=z(N, M, Hkv, D), v=z(N, M, Hkv, D), parent=z(N, M, dt=torch.int32), pos=z(N, dt=torch.int32),
                accepted=z(N, dt=torch.int32), kr=z(N, Hkv, W, D), vr=z(N, Hkv, W, D), state=z(N, Hkv, D, D, dt=torch.float32),
                kc=codes(D, torch.float8_e4m3fn), ks=codes(D // 32, torch.float8_e8m0fnu), vc=codes(D, torch.float8_e4m3fn),
                vs=codes(D // 32, torch.float8_e8m0fnu))


def test_host_tensors_are_refused():
    t = tensors()
    with pytest.raises(ValueError, match="contiguous device tensor"):
        rb.rattn_ring_pack(t["kr"], t["vr"])
    with pytest.raises(ValueError, match="contiguous device tensor"):
        rb.rattn_ring_unpack(t["kc"], t["ks"], t["vc"], t["vs"])
    with pytest.raises(ValueError, match="contiguous device tensor"):
        rb.rattn_decode_step_packed(t["q"][:, 0].contiguous(), t["k"][:, 0].contiguous(), t["v"][:, 0].contiguous(), t["pos"], t["kc"],
                                    t["ks"], t["vc"], t["vs"], t["state"])
    with pytest.raises(ValueError, match="contiguous device tensor"):
        rb.rattn_tree_step(t["q"], t["k"], t["v"], t["parent"], t["pos"], t["kr"], t["vr"], t["state"])
    with pytest.raises(ValueError, match="contiguous device tensor"):
        rb.rattn_tree_commit(t["k"], t["v"], t["parent"], t["accepted"], t["pos"], t["kr"], t["vr"], t["state"])


def test_the_host_layer_is_clean_under_asan_and_ubsan(tmp_path):
    """csrc/api.hip, plan.hip and cache_api.hip as plain C++ with stub launchers (as tests/test_host_sanitizers.py does it)."""
    gxx, rocm = shutil.which("g++"), "/opt/rocm"
    if not gxx or not os.path.exists(os.path.join(rocm, "include", "hip", "hip_runtime.h")):
        pytest.skip("g++ or the HIP headers are not available")
    exe = str(tmp_path / "cache_host_check")
    csrc, host = os.path.join(ROOT, "paper_2506_15545_amd", "csrc"), os.path.join(ROOT, "tests", "host")
    cmd = [gxx, "-x", "c++", "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-D__align__(n)=__attribute__((aligned(n)))",
           "-DHIP_SYMBOL(x)=(&x)", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-w",
           "-I", os.path.join(rocm, "include"), "-I", os.path.join(ROOT, "include"), "-I", csrc]
    cmd += [os.path.join(csrc, f) for f in ("api.hip", "plan.hip", "cache_api.hip")]
    cmd += [os.path.join(host, f) for f in ("stub_kernels.cpp", "stub_cache_kernels.cpp", "cache_host_check.cpp")]
    cmd += ["-L", os.path.join(rocm, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(rocm, "lib"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and "ALL OK" in r.stdout, r.stdout[-3000:] + r.stderr[-3000:]
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]
