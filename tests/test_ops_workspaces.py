"""Workspaces of the caller in the 4-bit product and the linear layer: the host layer run against the
stand-in for the HIP runtime of host_api.py (no GPU), and the refusals of the C ABI and the binding."""
import os
import subprocess

import pytest
import torch

import host_api
from paper_2601_16294_amd import sfcops as so
from test_ops_routes import STUBS

MAIN = r'''
int main() {
  char cmd[16];
  void *A = (void*)0x1000, *B = (void*)0x2000, *C = (void*)0x3000, *S = (void*)0x4000;
  unsigned long ws, wb, s;
  long M, N, K, out;
  while (scanf("%15s", cmd) == 1) {
    int rc = 0;
    if (!strcmp(cmd, "capture")) {
      if (scanf("%lu %ld", &s, &M) != 2) return 1;
      if (M) capturing.insert((hipStream_t)s);
      else capturing.erase((hipStream_t)s);
    } else {
      if (scanf("%ld %ld %ld %ld %lu %lu %lu", &M, &N, &K, &out, &ws, &wb, &s) != 7) return 1;
      const long q = (K + 31) / 32 * 16, z = (q / 16 + 3) / 4 * 4;
      if (!strcmp(cmd, "gemm")) rc = sfc_gemm_mx4_ws_ex(M, N, K, A, q, S, z, B, q, S, z, C, N, (int)out, (void*)ws, wb, (void*)s);
      else if (!strcmp(cmd, "linear")) rc = sfc_mx4_linear_ws(M, N, K, A, K, 1, B, q, S, z, C, N, (int)out, (void*)ws, wb, (void*)s);
      else if (!strcmp(cmd, "gemmsize")) printf("size n=%zu\n", sfc_gemm_mx4_ws_size(M, N, K, (int)out));
      else if (!strcmp(cmd, "linearsize")) printf("size n=%zu\n", sfc_mx4_linear_ws_size(M, N, K, (int)out));
      else return 1;
    }
    printf("ret rc=%d\n", rc);
  }
  return 0;
}
'''
WS = 1 << 36
MEMORY = ("malloc", "malloc_async", "malloc_in_graph", "free")


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("ops_workspaces"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    main, out = os.path.join(d, "main.cpp"), os.path.join(d, "ops_workspaces")
    with open(main, "w") as f:
        f.write(host_api.MAIN.split("int main()")[0] + STUBS.split("int main()")[0] + MAIN)
    src = [f"{host_api.CSRC}/{n}" for n in ("sfcgemm_api.cpp", "sfc_model.cpp", "sfc_ops_api.cpp")]
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", f"-I{d}", f"-I{host_api.ROOT}/include", f"-I{host_api.CSRC}", main,
                    *src, "-o", out], check=True)
    return out


def size(exe, entry, M, N, K, out):
    events, = host_api.run(exe, [f"{entry}size {M} {N} {K} {out} 0 0 1"])
    return dict(events)["size"]["n"]


def memory(events):
    """What a call allocated, curve tables left out."""
    return [(n, e) for n, e in events if n in MEMORY and e.get("n", 0) > 4096]


# (M, N, K): layers of K; one layer; few rows, converted by the product or by a launch before it
SHAPES = [(130, 70, 8192), (1000, 900, 16352), (500, 500, 512), (40, 100, 128), (4, 4096, 4096), (16, 14336, 4096), (4, 4096, 4128)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("out", [0, 1])
@pytest.mark.parametrize("entry", ["gemm", "linear"])
def test_calls_use_the_callers_memory_only(exe, entry, M, N, K, out):
    n = size(exe, entry, M, N, K, out)
    # every range that the call uses lies inside it, and all of it is used
    events, = host_api.run(exe, [f"{entry} {M} {N} {K} {out} {WS} {n} 1"])
    assert events[-1] == ("ret", {"rc": 0}) and memory(events) == []
    e = dict(events)
    ends = [0]
    if "quant" in e:
        assert e["quant"]["Q"] == WS and WS + M * e["quant"]["ldq"] <= e["quant"]["S"]
        ends.append(-(-(e["quant"]["S"] - WS + M * e["quant"]["lds"]) // 16) * 16)
    if "reduce" in e:
        assert e["tile"]["C"] == e["reduce"]["W"] >= WS + ends[-1]
        ends.append(e["tile"]["C"] - WS + e["tile"]["layers"] * M * N * 4)
    assert ends[-1] == n
    if n:
        events, = host_api.run(exe, [f"{entry} {M} {N} {K} {out} {WS} {n - 1} 1"])
        assert events == [("ret", {"rc": -3})]
        # none given: as many bytes of library memory
        events, = host_api.run(exe, [f"{entry} {M} {N} {K} {out} 0 0 1"])
        assert [e["n"] for name, e in events if name == "malloc_async"] == [n]
    events, = host_api.run(exe, [f"{entry} {M} {N} {K} {out} {WS + 8} {n + 8} 1"])
    assert events == [("ret", {"rc": -2})]


@pytest.mark.parametrize("entry", ["gemm", "linear"])
def test_graphs_of_one_stream_with_memory_of_their_own(exe, entry):
    """Recorded one after the other on one stream: nothing that either writes belongs to the other."""
    M, N, K = 130, 70, 8192
    n = size(exe, entry, M, N, K, 0)
    other = WS + n
    calls = host_api.run(exe, ["capture 1 1", f"{entry} {M} {N} {K} 0 {WS} {n} 1", "capture 1 0",
                               "capture 1 1", f"{entry} {M} {N} {K} 0 {other} {n} 1", "capture 1 0"])
    for ws, events in ((WS, calls[1]), (other, calls[4])):
        assert events[-1] == ("ret", {"rc": 0}) and memory(events) == []
        written = [e[k] for name, e in events for k in ("Q", "S", "W") if name in ("quant", "reduce") and k in e]
        assert written and all(ws <= p < ws + n for p in written)
    # without a workspace both use the stream's
    calls = host_api.run(exe, ["capture 1 1", f"{entry} {M} {N} {K} 0 0 0 1", "capture 1 0",
                               "capture 1 1", f"{entry} {M} {N} {K} 0 0 0 1", "capture 1 0"])
    assert dict(calls[1])["reduce"]["W"] == dict(calls[4])["reduce"]["W"]


@pytest.mark.parametrize("line", ["gemmsize -1 70 8192 0", "gemmsize 130 70 8191 0", "gemmsize 130 70 8192 2", "gemmsize 0 70 8192 0",
                                  "linearsize 130 -1 8192 0", "linearsize 130 0 8192 0", "linearsize 130 70 8192 7"])
def test_sizes_that_need_nothing(exe, line):
    events, = host_api.run(exe, [line + " 0 0 1"])
    assert events[0] == ("size", {"n": 0})


def test_binding_checks(monkeypatch):
    q = lambda r, c: so.mx4_empty(r, c, device="cpu")
    y = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="must be a CUDA tensor"):
        so._memory(torch.zeros(4), "test")
    with pytest.raises(TypeError, match="workspace must be a torch.Tensor"):
        so._memory(4096, "test")
    monkeypatch.setattr(so, "_tensor", lambda t, name, what: None)
    for bad in (torch.zeros(8, 8)[:, :4], torch.zeros(64)[::2]):
        for f in (lambda: so.sfc_gemm_mx4_ex(*q(4, 64), *q(8, 64), y, workspace=bad),
                  lambda: so.sfc_mx4_linear(torch.zeros(4, 64), *q(8, 64), y, workspace=bad)):
            with pytest.raises(ValueError, match="contiguous"):
                f()
    t = torch.zeros(6)
    assert so._memory(t, "test") == (t.data_ptr(), 24)
    # an empty workspace is not "none": a call that needs memory refuses it
    assert so._memory(torch.zeros(0), "test") == (16, 0)
