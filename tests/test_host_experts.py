"""The host side of the router's, the experts' and the 4-bit rows' entry points, without a GPU: the grids and workspaces of
every call over the documented ranges (tests/host_sanitize/launch_shapes_experts.cpp), and every refusal with the checks'
host code under AddressSanitizer and UndefinedBehaviorSanitizer (tests/host_sanitize/abi_errors_experts.cpp)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FLAGS = ["--offload-arch=gfx950", "-O1", "-std=c++17", "-Wno-inline-asm", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _objects(names):
    from paper_2411_08446_amd import build
    objs = [os.path.join(build.BUILD_DIR, n + ".o") for n in names]
    if not all(os.path.exists(o) for o in objs):
        build.build(verbose=False)
    return objs


def _run(command, timeout=600):
    res = subprocess.run(command, capture_output=True, text=True, timeout=timeout)
    assert res.returncode == 0, res.stdout + res.stderr
    return res


def test_launches_over_the_documented_ranges(tmp_path):
    from paper_2411_08446_amd import build
    objs = _objects([os.path.splitext(s)[0] for s in build.SOURCES])
    exe = str(tmp_path / "launches")
    _run([build.HIPCC, *FLAGS, "-c", os.path.join(ROOT, "tests", "host_sanitize", "launch_shapes_experts.cpp"), "-o", exe + ".o"])
    _run([build.HIPCC, "--offload-arch=gfx950", exe + ".o", *objs, "-o", exe])
    assert " 0 failures" in _run([exe], timeout=120).stdout


def test_refusals_are_clean_under_asan_and_ubsan(tmp_path):
    from paper_2411_08446_amd import build
    own = ["api", "api_experts"]
    others = _objects([os.path.splitext(s)[0] for s in build.SOURCES if os.path.splitext(s)[0] not in own])
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined"]
    objs = []
    for src in [os.path.join(build.CSRC, o + ".hip") for o in own] + [os.path.join(ROOT, "tests", "host_sanitize", "abi_errors_experts.cpp")]:
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        _run([build.HIPCC, *FLAGS, "-g", *san, "-c", src, "-o", objs[-1]])
    exe = str(tmp_path / "refusals")
    _run([build.HIPCC, "--offload-arch=gfx950", *san, *objs, *others, "-o", exe])
    res = _run([exe], timeout=120)
    assert res.stdout.startswith("0 failures"), res.stdout
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr
