"""The layout of the layer operators' products in any workspace that a call accepts, on the CPU: tests/hostmath/layers_driver.cpp under
AddressSanitizer and UBSan, and the calls through the host build of the library."""
import os
import subprocess

import pytest
import torch

import paper_2602_12630_amd as T
from test_layers_host import emu, mat, ws  # noqa: F401

HERE = os.path.dirname(os.path.abspath(__file__))


def test_plans_fit_into_their_workspace(tmp_path):
    exe = str(tmp_path / "layers_driver")
    cmd = ["g++", "-O1", "-g", "-std=c++17", "-DTC_HOST_EMU", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           "-static-libasan", "-o", exe, os.path.join(HERE, "hostmath", "layers_driver.cpp")]
    built = subprocess.run(cmd, capture_output=True, text=True)
    err = built.stderr.lower()
    if built.returncode != 0 and "cannot find" in err and ("asan" in err or "ubsan" in err or "sanitize" in err):
        pytest.skip("the sanitizer runtimes are not installed")
    assert built.returncode == 0, built.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    if "ASan runtime does not come first" in run.stderr:
        pytest.skip("a preloaded library keeps the sanitizer runtime from starting here")
    assert run.returncode == 0, (run.stdout + run.stderr)[-4000:]
    assert "layers driver: ok" in run.stdout


@pytest.mark.parametrize("most,rows,k,n", [(16384, 1, 1024, 1), (16384, 64, 1024, 8), (256, 32, 2048, 1024)])
def test_a_workspace_of_many_rows_serves_fewer(emu, most, rows, k, n):  # noqa: F811
    """also where the fewer rows would like more of it"""
    emu.linear(mat(rows, k), mat(n, k), mat(rows, n), workspace=ws(emu.linear_workspace(most, k, n)))
    emu.linear_backward(mat(rows, n), mat(rows, k), mat(n, k), dx=mat(rows, k), dw=mat(n, k), workspace=ws(emu.linear_backward_workspace(most, k, n)))


@pytest.mark.parametrize("rows,cols", [(1023, 512), (1023, 8), (600, 100)])
def test_a_workspace_of_many_rows_serves_the_norm_of_fewer(emu, rows, cols):  # noqa: F811
    m, v = mat(rows, cols), torch.zeros(rows)
    for most in (rows, 1024, 1500, 16384):
        emu.norm_backward(0, m, m, None, v, v, m, torch.zeros(cols), torch.zeros(cols), ws(emu.norm_backward_workspace(most, cols)))


def test_a_workspace_that_is_too_small_is_refused(emu):  # noqa: F811
    m, w = mat(300, 1024), mat(8, 1024)
    dy = mat(300, 8)
    least = emu.linear_backward_workspace(300, 1, 8)          # (an inner width of one needs no room for products)
    emu.linear_backward(dy, m, w, dx=mat(300, 1024), dw=mat(8, 1024), workspace=ws(least))
    for bad in (None, ws(least - 1), ws(least + 16)[8:]):
        with pytest.raises(T.TcError) as e:
            emu.linear_backward(dy, m, w, dx=mat(300, 1024), dw=mat(8, 1024), workspace=bad)
        assert e.value.code == T.binding.TC_ERR_ARG
    room = emu.linear_workspace(300, 1024, 8)
    assert room > 0
    with pytest.raises(T.TcError):
        emu.linear(m, w, mat(300, 8), workspace=ws(room + 16)[8:])
