"""The host code of the serving loop's entry points under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only, no GPU):
`csrc/api.hip` with the sanitizers on its host side, linked with a driver whose every call is refused, and the ordinary kernel objects."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2407_07304_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def test_serving_entry_points_are_clean_under_host_sanitizers(tmp_path):
    from paper_2407_07304_amd import build
    kernels = [os.path.join(CSRC, s.replace(".hip", ".o")) for s in build.SOURCES if s != "api.hip"]
    if not all(os.path.exists(o) for o in kernels):
        build.build()
    api_o, drv_o, exe = (str(tmp_path / n) for n in ("api_san.o", "driver_san.o", "serving_abi_sanitize_driver"))
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                "-Xarch_host", "-fno-sanitize-recover=all"]

    def run(cmd, **more):
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, **more)
        assert r.returncode == 0, r.stdout[-4000:]
        return r.stdout

    run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC"] + host_san +
        ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-c", os.path.join(CSRC, "api.hip"), "-o", api_o])
    run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-c",
         os.path.join(HERE, "host_models", "serving_abi_sanitize_driver.cpp"), "-o", drv_o])
    run([HIPCC, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address,undefined", api_o, drv_o] + kernels + ["-o", exe])
    # (leak detection off: the HIP runtime keeps its own allocations until the process ends)
    assert "clean" in run([exe], timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1"))
