"""The validation of lsh_qk.h's and lsh_cache.h's entry points (host code) under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU, at the ends of the sizes they take and past them."""
import glob
import os
import shutil
import subprocess

import pytest

from test_sanitizers import PKG, ROOT, _run


def test_validation_under_sanitizers(tmp_path):
    objs = [os.path.join(PKG, "_build", f + ".o") for f in ("hash", "sort", "attn_fwd", "attn_bwd", "combine", "dense",
                                                            "block", "lsh_api", "block_api", "qk", "cache", "cache_attn")]
    if not all(os.path.exists(o) for o in objs):
        pytest.skip("kernel objects not built (run __graft_entry__.build())")
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    rt = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    if not os.path.exists(hipcc) or not rt:
        pytest.skip("hipcc or the clang sanitizer runtime is missing")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined"]
    api = []
    for src in ("qk_api.cpp", "cache_api.cpp"):
        o = str(tmp_path / (src + ".san.o"))
        subprocess.check_call([hipcc, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", *san,
                               "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "csrc"),
                               "-c", os.path.join(PKG, "csrc", src), "-o", o])
        api.append(o)
    lib = str(tmp_path / "liblsh_san.so")
    subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *san, "-shared-libasan", *api, *objs,
                           "-o", lib])
    res = _run(f"""
        import ctypes, itertools
        from paper_2001_04451_amd import cache, lsh, qk
        lsh.LIB_PATH = {lib!r}
        F = ctypes.c_void_p(0x1000)
        big = [0, 1, 7, 16, 64, 1024, 4096, 2 ** 14, 2 ** 20, 2 ** 30, 2 ** 31 - 1, -1, -2 ** 31]
        wide = big + [2 ** 31, 2 ** 40, 2 ** 62, -2 ** 62]
        for f, vals in (("T", wide), ("L", wide), ("x_stride", wide), ("dx_stride", wide), ("Hq", big), ("Hk", big),
                        ("d", big), ("rot", big)):
            for x in vals:
                c = qk.QkConfigC(6, 3, 0, 0, 2, 1, 64, 64, 0, 0, 1e-6)
                setattr(c, f, x)
                n = qk.lib().lsh_qk_workspace_bytes(ctypes.byref(c))
                # no launch: without x the call is refused whatever the configuration
                assert qk.lib().lsh_qk_norm_rotate_fwd(ctypes.byref(c), 1, None, F, F, F, F, F, F, None) in (-1, -2)
                assert qk.lib().lsh_qk_norm_rotate_bwd(ctypes.byref(c), 1, F, F, F, F, F, F, F, F, F, F, F,
                                                       max(n, 1) - 1, None) in (-1, -2)
        P, S = cache.CachePagesC(*[0x1000] * 5), cache.CacheSeqsC(*[0x1000] * 3)
        names = [f for f, _ in cache.CacheConfigC._fields_[:14]]
        for f, g in itertools.product(names, names):
            for x, y in itertools.product(wide if f in names[:4] else big, [None, 1, 2 ** 31 - 1]):
                c = cache.CacheConfigC(8, 0, 0, 0, 3, 4, 2, 64, 16, 10, 4, 1, 0, 0, 0.125, 1e5)
                setattr(c, f, x)
                if y is not None:
                    setattr(c, g, y)
                n = cache.lib().lsh_cache_workspace_bytes(ctypes.byref(c))
                head = (ctypes.byref(c), 1, ctypes.byref(P), ctypes.byref(S))
                assert cache.lib().lsh_cache_write(*head, None, F, None) in (-1, -2)
                assert cache.lib().lsh_cache_read(*head, None, None, None) in (-1, -2)
                assert cache.lib().lsh_cache_attn_fwd(*head, F, F, F, F, max(n, 1) - 1, None) in (-1, -2)
        print("ok")
    """, {"LD_PRELOAD": rt[0]})
    assert res.returncode == 0 and "ok" in res.stdout, res.stdout[-3000:] + res.stderr[-3000:]
    assert "runtime error" not in res.stderr and "ERROR: AddressSanitizer" not in res.stderr
