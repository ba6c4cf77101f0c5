"""Which kernel, grid and memory a call of the 4-bit and expert operators takes: the host
layer run against the stand-in for the HIP runtime of host_api.py, so no GPU is needed."""
import os
import subprocess

import pytest

import host_api
from mx4_cases import DEPTHS, EXPERTS, PRODUCTS

STUBS = r'''
#include "sfc_ops_params.h"
namespace sfc {
static unsigned long v(const void* p) { return (unsigned long)(uintptr_t)p; }
hipError_t launch_mx4_quant(const Mx4QuantParams& p, bool bf16, int, hipStream_t) {
  printf("quant rows=%ld cols=%ld bf16=%d Q=%lu S=%lu ldq=%ld lds=%ld\n", (long)p.rows, (long)p.cols, (int)bf16, v(p.Q), v(p.S),
         (long)p.ldq, (long)p.lds);
  return hipSuccess;
}
hipError_t launch_mx4_dequant(const Mx4DequantParams&, bool, int, hipStream_t) { return hipSuccess; }
static hipError_t tile(int b, const Mx4GemmParams& p, Mx4Mode mode, bool bf16, int grid) {
  printf("tile b=%d mode=%d bf16=%d grid=%d layers=%d C=%lu A=%lu As=%lu K=%ld table=%lu gm=%d gn=%d\n", b, (int)mode, (int)bf16,
         grid, p.layers, v(p.C), v(p.A), v(p.As), (long)p.K, v(p.table), p.gm, p.gn);
  return hipSuccess;
}
hipError_t launch_mx4_256x256(const Mx4GemmParams& p, Mx4Mode m, bool b, int g, hipStream_t) { return tile(256, p, m, b, g); }
hipError_t launch_mx4_128x128(const Mx4GemmParams& p, Mx4Mode m, bool b, int g, hipStream_t) { return tile(128, p, m, b, g); }
hipError_t launch_mx4_rows(const Mx4GemmParams& p, Mx4Mode mode, int fm, bool narrow, bool, hipStream_t) {
  printf("rows fm=%d narrow=%d mode=%d\n", fm, (int)narrow, (int)mode);
  return hipSuccess;
}
hipError_t launch_mx4_few(const Mx4GemmParams& p, Mx4Rows rows, int, bool, hipStream_t) {
  printf("few rows=%d M=%ld K=%ld X=%lu x_cols=%ld\n", (int)rows, (long)p.M, (long)p.K, v(p.X), (long)p.x_cols);
  return hipSuccess;
}
hipError_t launch_moe_sort(const MoeSortParams& p, hipStream_t) {
  printf("sort counts=%lu\n", v(p.counts));
  return hipSuccess;
}
hipError_t launch_moe_dispatch(const MoeRowsParams&, bool, int, hipStream_t) { return hipSuccess; }
hipError_t launch_moe_combine(const MoeRowsParams&, bool, int, hipStream_t) { return hipSuccess; }
hipError_t launch_moe_combine_grad(const MoeRowsParams&, bool, int, hipStream_t) { return hipSuccess; }
}  // namespace sfc
int main() {
  char cmd[16];
  void *A = (void*)0x1000, *B = (void*)0x2000, *C = (void*)0x3000, *S = (void*)0x4000;
  while (scanf("%15s", cmd) == 1) {
    int rc = 0;
    long a, b, c, d, e;
    unsigned long s;
    if (!strcmp(cmd, "capture")) {
      if (scanf("%lu %ld", &s, &a) != 2) return 1;
      if (a) capturing.insert((hipStream_t)s);
      else capturing.erase((hipStream_t)s);
    } else {
      if (scanf("%ld %ld %ld %ld %ld %lu", &a, &b, &c, &d, &e, &s) != 6) return 1;
      void* st = (void*)s;
      const long q = (c + 31) / 32 * 16, z = (q / 16 + 3) / 4 * 4;
      if (!strcmp(cmd, "gemm")) rc = sfc_gemm_mx4_ex(a, b, c, A, q, S, z, B, q, S, z, C, b, (int)d, st);
      else if (!strcmp(cmd, "linear")) rc = sfc_mx4_linear(a, b, c, A, c, (int)e, B, q, S, z, C, b, (int)d, st);
      else if (!strcmp(cmd, "experts")) rc = sfc_moe_gemm_mx4_ex(a, b, c, (int)e, A, q, S, z, B, q, b * q, S, z, b * z, (int*)S, C, b, (int)d, st);
      else if (!strcmp(cmd, "depth")) rc = sfc_moe_wgrad_mx4_ex(a, b, c, (int)e, A, q, S, z, B, q, S, z, (int*)S, C, b, a * b, (int)d, st);
      else if (!strcmp(cmd, "sort")) rc = sfc_moe_sort(a, (int)b, (int)c, (int*)A, d, (int*)B, (int*)C, (int*)S, nullptr, 0, st);
      else return 1;
    }
    printf("ret rc=%d\n", rc);
  }
  return 0;
}
'''


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("ops_routes"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    main, out = os.path.join(d, "main.cpp"), os.path.join(d, "ops_routes")
    with open(main, "w") as f:
        f.write(host_api.MAIN.split("int main()")[0] + STUBS)
    src = [f"{host_api.CSRC}/{n}" for n in ("sfcgemm_api.cpp", "sfc_model.cpp", "sfc_ops_api.cpp")]
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", f"-I{d}", f"-I{host_api.ROOT}/include", f"-I{host_api.CSRC}", main,
                    *src, "-o", out], check=True)
    return out


def route(events):
    assert events[-1] == ("ret", {"rc": 0})
    for name, e in events:
        if name == "few":
            turns = -(-e["K"] // 512)
            waves = 4 if turns <= 4 else 8
            return f"few{1 if turns <= waves else 2 if turns <= 2 * waves else 4}"
        if name == "rows":
            return f"rows{e['fm']}" + ("n" if e["fm"] == 1 and e["narrow"] else "")
        if name == "tile":
            return str(e["b"]) + (f"/{e['layers']}" if e["layers"] > 1 else "")
    return None


@pytest.mark.parametrize("shape,want", PRODUCTS)
@pytest.mark.parametrize("out", [0, 1])
def test_products_reach_their_kernels(exe, shape, want, out):
    M, N, K = shape
    events, = host_api.run(exe, [f"gemm {M} {N} {K} {out} 0 1"])
    assert route(events) == want
    for name, e in events:
        if name == "tile":
            b = e["b"]
            assert e["gm"] == -(-M // b) and e["gn"] == -(-N // b) and e["table"] != 0
            assert 1 <= e["grid"] <= min(e["gm"] * e["gn"] * e["layers"], 256 if b == 256 else 512)
            # layer copies are fp32, in memory of their own, and a reduction follows
            assert (e["layers"] == 1) == (e["C"] == 0x3000) == ("reduce" not in dict(events))
            assert e["bf16"] == (1 if out and e["layers"] == 1 else 0)


@pytest.mark.parametrize("case,want", EXPERTS)
@pytest.mark.parametrize("out", [0, 1])
def test_experts_reach_their_kernels(exe, case, want, out):
    counts, N, K = case
    rows = max(sum(counts), 5)
    events, = host_api.run(exe, [f"experts {rows} {N} {K} {out} {len(counts)} 1"])
    assert route(events) == want
    for name, e in events:
        if name == "tile":
            assert e["mode"] == 1 and 1 <= e["grid"] <= (256 if e["b"] == 256 else 512)


@pytest.mark.parametrize("case,want", DEPTHS)
@pytest.mark.parametrize("out", [0, 1])
def test_weight_gradients_reach_their_kernels(exe, case, want, out):
    starts, M, N = case
    events, = host_api.run(exe, [f"depth {M} {N} {starts[-1] + 31} {out} {len(starts) - 1} 1"])
    assert route(events) == want


@pytest.mark.parametrize("M,N,K,launches", [(1, 4096, 4096, ["few"]), (8, 14336, 4096, ["few"]), (16, 8192, 4000, ["few"]),
                                            (16, 14336, 4096, ["quant", "few"]), (4, 4096, 4128, ["quant", "few"]),
                                            (40, 100, 100, ["quant", "rows"]), (500, 500, 500, ["quant", "tile"])])
def test_linear_launches(exe, M, N, K, launches):
    events, = host_api.run(exe, [f"linear {M} {N} {K} 1 1 1"])
    assert [n for n, _ in events if n in ("quant", "few", "rows", "tile", "reduce")] == launches
    for name, e in events:
        if name == "few":
            assert (e["rows"] == 1) == (launches == ["few"]) and e["x_cols"] == (K if launches == ["few"] else 0)
            assert e["K"] == -(-K // 32) * 32


def test_linear_memory_holds_codes_scales_and_copies(exe):
    M, N, K = 130, 70, 8190
    events, = host_api.run(exe, [f"linear {M} {N} {K} 0 1 1"])
    e = dict(events)
    base, size = e["malloc_async"]["p"], e["malloc_async"]["n"]
    q, t, r = e["quant"], e["tile"], e["reduce"]
    blocks = -(-K // 32)
    assert q["ldq"] == 16 * blocks and q["lds"] % 4 == 0 and q["lds"] >= blocks
    assert q["Q"] == base == t["A"] and q["S"] == t["As"] and q["Q"] % 16 == 0 and q["S"] % 4 == 0
    assert q["Q"] + M * q["ldq"] <= q["S"] and q["S"] + M * q["lds"] <= t["C"] == r["W"] and t["C"] % 16 == 0
    assert t["layers"] == r["layers"] > 1 and t["C"] + t["layers"] * M * N * 4 <= base + size


def test_recorded_calls_own_their_memory(exe):
    line = "linear 130 70 8190 0 1 1"
    calls = host_api.run(exe, [line, "capture 1 1", line, "capture 1 0", line, "linear 900 70 8190 0 1 1"])
    eager, rec, again, larger = calls[0], calls[2], calls[4], calls[5]
    at = lambda ev: dict(ev)["quant"]["Q"]
    assert at(eager) == at(again) != at(rec)
    assert "malloc" in dict(rec) and "malloc_async" not in dict(rec) and "malloc_in_graph" not in dict(rec)
    # the larger call frees the eager memory, never the recorded one
    assert [e["p"] for n, e in larger if n == "free"] == [at(eager)]
    assert [x for x in rec if x[0] == "free"] == []


def test_streams_have_memory_of_their_own(exe):
    a, b = host_api.run(exe, ["linear 130 70 8190 0 1 1", "linear 130 70 8190 0 1 2"])
    assert dict(a)["quant"]["Q"] != dict(b)["quant"]["Q"]


@pytest.mark.parametrize("slots,E,need", [(4096, 8, 0), (4097, 8, 2 * 8 * 4), (70000, 1024, 18 * 1024 * 4)])
def test_sort_memory(exe, slots, E, need):
    events, = host_api.run(exe, [f"sort {slots} {E} 1 {slots} 0 1"])
    got = [e["n"] for n, e in events if n == "malloc_async"]
    assert got == ([need] if need else []) and events[-1] == ("ret", {"rc": 0})
