"""A host-side AddressSanitizer + UndefinedBehaviorSanitizer build of the key/value cache's validation, workspace sizes and layout (CPU only,
no GPU code runs; hipcc: each -fsanitize= directly after -Xarch_host)."""
import os
import tempfile
from concurrent.futures import ThreadPoolExecutor

from test_sanitizers_cpu import ENV, SAN, _run


def test_kv_cache_validation_under_host_sanitizers():
    from paper_2601_12150_amd import build as hip_build
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = [f for f in hip_build.FLAGS if f != "-O3"] + ["-O1"]
    clang = os.path.join(os.path.dirname(hip_build.HIPCC), "amdclang++")
    with tempfile.TemporaryDirectory() as tmp:
        def compile_one(src):
            obj = os.path.join(tmp, src.replace(".hip", ".o"))
            # (the cache's sources under the sanitizers; the others, which the error messages and the count of compute units come with, as they are)
            built = os.path.join(hip_build.OBJ, os.path.basename(obj))
            if not src.startswith("ns_kv") and os.path.exists(built):
                return built
            rc, out = _run([hip_build.HIPCC, *flags, *(san if src.startswith("ns_kv") else []), "-c", os.path.join(hip_build.CSRC, src), "-o", obj])
            assert rc == 0, out
            return obj
        with ThreadPoolExecutor(max_workers=8) as ex:
            objs = list(ex.map(compile_one, hip_build.SOURCES))
        drv, exe = os.path.join(tmp, "kv_abi_driver.o"), os.path.join(tmp, "kv_abi_san")
        rc, out = _run([clang, "-O1", "-g", "-std=c++17", "-fsanitize=address", "-fsanitize=undefined", "-fno-omit-frame-pointer", "-c",
                        os.path.join(SAN, "kv_abi_driver.cpp"), "-o", drv])
        assert rc == 0, out
        rc, out = _run([hip_build.HIPCC, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-o", exe, drv, *objs])
        assert rc == 0, out
        rc, out = _run([exe], env=ENV)
        assert rc == 0 and "key/value cache sanitizer run ok" in out, out
        assert "ERROR: AddressSanitizer" not in out and "runtime error" not in out, out
