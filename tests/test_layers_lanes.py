"""The layer operators' kernels and launches on the CPU, lane by lane under AddressSanitizer and UBSan's checks of alignment, bounds and overflow (tests/hostmath/layers_lanes.cpp): every address
that they form lies in its block, every output entry is written, and the tiles of the products hold what belongs there."""
import os
import subprocess

import pytest

from test_host_logic import ROOT

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "hostmath")
CLANG = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")


def test_layer_kernels_stay_inside_their_buffers(tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("the kernels' vector types want clang")
    exe = str(tmp_path / "layers_lanes")
    cmd = [CLANG, "-x", "c++", "-O1", "-gline-tables-only", "-std=c++17", "-fsanitize=address,alignment,bounds,signed-integer-overflow",
           "-fno-sanitize-recover=all", "-ftrivial-auto-var-init=zero", "-Wno-everything", "-I", os.path.join(HERE, "lanes"), "-o", exe, os.path.join(HERE, "layers_lanes.cpp")]
    built = subprocess.run(cmd, capture_output=True, text=True, cwd=ROOT)
    if built.returncode != 0 and "libclang_rt" in built.stderr:
        pytest.skip("the sanitizer runtimes are not installed")
    assert built.returncode == 0, built.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=900)
    if "ASan runtime does not come first" in run.stderr:
        pytest.skip("a preloaded library keeps the sanitizer runtime from starting here")
    assert run.returncode == 0, (run.stdout + run.stderr)[-6000:]
    assert "layers lanes: ok" in run.stdout
