"""The validation of lsh_w4.h's, lsh_residual.h's and the append's entry points (host code) under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU, at the ends of the sizes they take and past them."""
import glob
import os
import shutil
import subprocess

import pytest

from test_sanitizers import PKG, ROOT, _run


def test_validation_under_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    rt = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    apis = ("w4_api", "residual_api", "cache_api")
    objs = [o for o in sorted(glob.glob(os.path.join(PKG, "_build", "*.o"))) if os.path.basename(o)[:-2] not in apis]
    if len(objs) < 15 or not os.path.exists(hipcc) or not rt:
        pytest.skip("kernel objects not built (run __graft_entry__.build()), or hipcc or the sanitizer runtime is missing")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined"]
    built = []
    for src in apis:
        o = str(tmp_path / (src + ".san.o"))
        subprocess.check_call([hipcc, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", *san,
                               "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
                               "-c", os.path.join(PKG, "csrc", src + ".cpp"), "-o", o])
        built.append(o)
    lib = str(tmp_path / "liblsh_san.so")
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *san, "-shared-libasan", *built, *objs,
                           "-o", lib])
    res = _run(f"""
        import ctypes, itertools
        from paper_2001_04451_amd import cache, lsh, qk, residual, w4
        lsh.LIB_PATH = {lib!r}
        F = ctypes.c_void_p(0x1000)
        ref = ctypes.byref
        big = [0, 1, 7, 16, 32, 64, 1024, 4096, 2 ** 14, 2 ** 20, 2 ** 30, 2 ** 31 - 1, -1, -2 ** 31]
        wide = big + [2 ** 31, 2 ** 40, 2 ** 62, -2 ** 62]
        # no launch: a pointer that the call needs is missing whatever the configuration
        for f, g in itertools.product(("N", "K", "type", "group", "zeros"), repeat=2):
            for x, y in itertools.product(big, big):
                c = w4.W4ConfigC(48, 256, 0, 128, 0)
                setattr(c, f, x)
                setattr(c, g, y)
                assert w4.lib().lsh_w4_weight_bytes(ref(c)) >= 0
                assert w4.lib().lsh_w4_quantize(ref(c), 1, None, F, None) in (-1, -2)
                assert w4.lib().lsh_w4_pack(ref(c), F, None, F, F, None) in (-1, -2)
                assert w4.lib().lsh_w4_unpack(ref(c), 1, F, None, None) in (-1, -2)
        for N, K in ((48, 256), (1, 32), (2 ** 22, 32), (2 ** 16, 2 ** 17)):
            c = w4.W4ConfigC(N, K, 0, 128, 1)
            for M, stride in itertools.product(wide, wide):
                n = w4.lib().lsh_w4_workspace_bytes(ref(c), M)
                assert w4.lib().lsh_linear_w4(ref(c), M, None, stride, F, None, None, 1.0, 0, F, None, F, n, None) in (-1, -2)
        names = ("T", "f_stride", "gate_stride", "D", "norm", "post", "pre", "gate")
        W, G = residual.ResidualWeightsC(*[0x1000] * 5), residual.ResidualGradsC(0, *[0x1000] * 7)
        for f, g in itertools.product(names, names):
            for x, y in itertools.product(wide if f in names[:3] else big, wide if g in names[:3] else big):
                c = residual.ResidualConfigC(6, 0, 0, 64, 1, 1, 1, 2, 1.0, 1e-6)
                setattr(c, f, x)
                setattr(c, g, y)
                n = residual.lib().lsh_residual_workspace_bytes(ref(c))
                assert residual.lib().lsh_residual_norm_fwd(ref(c), 1, F, None, F, ref(W), None, F, None) in (-1, -2)
                assert residual.lib().lsh_residual_norm_bwd(ref(c), 1, F, F, F, ref(W), F, F, ref(G), F, n, None) in (-1, -2)
        P, S = cache.CachePagesC(*[0x1000] * 5), cache.CacheSeqsC(*[0x1000] * 3)
        for f in ("T", "L", "x_stride", "dx_stride", "Hq", "Hk", "d", "rot"):
            for g, y in itertools.product(("T", "H", "Hkv", "n_seq", "q_stride"), big):
                for x in wide if f in ("T", "L", "x_stride", "dx_stride") else big:
                    c = cache.CacheConfigC(8, 0, 0, 0, 3, 4, 2, 64, 16, 10, 4, 1, 0, 0, 0.125, 1e5)
                    k = qk.QkConfigC(8, 0, 0, 0, 4, 2, 64, 64, 0, 0, 1e-6)
                    setattr(c, g, y)
                    if hasattr(k, g):
                        setattr(k, g, y)
                    setattr(k, f, x)
                    assert cache.lib().lsh_cache_append(ref(c), ref(k), 1, ref(P), ref(S), None, F, F, F, F, None) in (-1, -2)
        print("ok")
    """, {"LD_PRELOAD": rt[0]})
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:] + res.stderr[-3000:]
    assert "runtime error" not in res.stderr and "ERROR: AddressSanitizer" not in res.stderr
