"""Which products store past the caches: outputs of 32 MB and more, but never layer copies, which are
read next.  The host layer run against the stand-in for the HIP runtime of host_api.py (no GPU)."""
import os
import subprocess

import pytest

import host_api
from test_ops_routes import STUBS


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("ops_past"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    stubs = STUBS.replace('printf("tile b=%d', 'printf("tile past=%d b=%d', 1).replace('gn=%d\\n", b, (int)mode', 'gn=%d\\n", (int)p.past, b, (int)mode', 1)
    assert stubs.count("past") == 2
    main, out = os.path.join(d, "main.cpp"), os.path.join(d, "ops_past")
    with open(main, "w") as f:
        f.write(host_api.MAIN.split("int main()")[0] + stubs)
    src = [f"{host_api.CSRC}/{n}" for n in ("sfcgemm_api.cpp", "sfc_model.cpp", "sfc_ops_api.cpp")]
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", f"-I{d}", f"-I{host_api.ROOT}/include", f"-I{host_api.CSRC}", main,
                    *src, "-o", out], check=True)
    return out


@pytest.mark.parametrize("line,past", [
    ("gemm 4096 4096 4096 1 0 1", 1), ("gemm 4096 4095 4096 1 0 1", 0), ("gemm 2048 4096 4096 0 0 1", 1), ("gemm 2047 4096 4096 0 0 1", 0),
    ("linear 4096 4096 4096 1 1 1", 1), ("linear 4095 4096 4096 1 0 1", 0),
    ("experts 4096 4096 1024 1 8 1", 1), ("experts 4095 4096 1024 1 8 1", 0), ("experts 2048 4096 1024 0 8 1", 1),
    ("depth 1024 2048 4096 1 8 1", 1), ("depth 1024 2047 4096 1 8 1", 0), ("depth 1024 1024 4096 0 8 1", 1), ("depth 1023 1024 4096 0 8 1", 0)])
def test_products(exe, line, past):
    events, = host_api.run(exe, [line])
    assert events[-1] == ("ret", {"rc": 0})
    tile = dict(events)["tile"]
    assert tile["past"] == past and tile["layers"] == 1


@pytest.mark.parametrize("out", [0, 1])
def test_layer_copies_stay(exe, out):
    events, = host_api.run(exe, [f"gemm 100 100 16384 {out} 0 1"])
    tile = dict(events)["tile"]
    assert tile["layers"] > 1 and tile["past"] == 0 and "reduce" in dict(events)
