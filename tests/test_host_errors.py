"""What the C boundary promises when the host's memory is used up (tests/hostmath/errors_driver.cpp, the host build of the library)."""
import os
import subprocess

from test_host_logic import ROOT

HERE = os.path.dirname(os.path.abspath(__file__))


def test_refusals_without_memory_for_their_message(tmp_path):
    exe, csrc = str(tmp_path / "errors_driver"), os.path.join(ROOT, "paper_2602_12630_amd", "csrc")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-DTC_HOST_EMU", "-DTC_FB_C=8", "-Wno-unknown-pragmas", "-o", exe,
                           os.path.join(HERE, "hostmath", "errors_driver.cpp"), os.path.join(csrc, "tc_lib.cpp"), os.path.join(csrc, "tc_layers.cpp")])
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout + run.stderr
    assert "errors driver: ok" in run.stdout
