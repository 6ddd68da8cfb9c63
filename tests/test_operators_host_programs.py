"""Host code of the operators around the layer that needs no device, compiled into small programs of its own: the bound of the scored
routing's first products (route_bounds_host.cpp)."""
import os
import subprocess

from paper_2512_17073_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def _run(tmp_path, source):
    obj, exe = str(tmp_path / "program.o"), str(tmp_path / "program")
    subprocess.run([build._hipcc(), "--cuda-host-only", "-std=c++17", "-O1", "-fPIC", "-x", "hip", "-c", source, "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe], check=True)     # (no HIP runtime)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_a_token_norm_is_bounded_from_above(tmp_path):
    _run(tmp_path, os.path.join(HERE, "route_bounds_host.cpp"))
