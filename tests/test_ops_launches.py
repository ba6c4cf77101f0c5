"""Long matrices are dealt to several launches, each below 2^32 threads, that cover every row, column
and token once: the host layer of the row operators run against the stand-in for the HIP runtime of
host_api.py, so no GPU is needed.

Threads of a launch (of the kernels in sfc_moe.hip and sfc_mx4_quant.hip): at most 256 for a row or
token, 256 for 16 rows to clear, 512 for 256 rows x 128 columns or 256 for 128 x 128."""
import os
import subprocess

import pytest

import host_api

STUBS = r'''
#include "sfc_ops_params.h"
namespace sfc {
static unsigned long v(const void* p) { return (unsigned long)(uintptr_t)p; }
hipError_t launch_mx4_quant(const Mx4QuantParams& p, bool bf16, int, hipStream_t) {
  printf("quant rows=%ld cols=%ld x_rows=%ld X=%lu order=%lu Q=%lu S=%lu Qt=%lu St=%lu\n", (long)p.rows, (long)p.cols, (long)p.x_rows,
         v(p.X), v(p.order), v(p.Q), v(p.S), v(p.Qt), v(p.St));
  return hipSuccess;
}
hipError_t launch_mx4_dequant(const Mx4DequantParams& p, bool, int, hipStream_t) {
  printf("dequant rows=%ld Q=%lu S=%lu Y=%lu\n", (long)p.rows, v(p.Q), v(p.S), v(p.Y));
  return hipSuccess;
}
hipError_t launch_mx4_256x256(const Mx4GemmParams&, Mx4Mode, bool, int g, hipStream_t) { printf("tile grid=%d\n", g); return hipSuccess; }
hipError_t launch_mx4_128x128(const Mx4GemmParams&, Mx4Mode, bool, int g, hipStream_t) { printf("tile grid=%d\n", g); return hipSuccess; }
hipError_t launch_mx4_rows(const Mx4GemmParams& p, Mx4Mode, int fm, bool, bool, hipStream_t) {
  printf("rows fm=%d N=%ld\n", fm, (long)p.N);
  return hipSuccess;
}
hipError_t launch_mx4_few(const Mx4GemmParams&, Mx4Rows, int, bool, hipStream_t) { printf("few n=1\n"); return hipSuccess; }
hipError_t launch_moe_sort(const MoeSortParams&, hipStream_t) { return hipSuccess; }
hipError_t launch_moe_dispatch(const MoeRowsParams& p, bool, int, hipStream_t) {
  printf("dispatch tokens=%ld rows=%ld X=%lu order=%lu weights=%lu Y=%lu\n", (long)p.tokens, (long)p.rows, v(p.X), v(p.order), v(p.weights), v(p.Y));
  return hipSuccess;
}
hipError_t launch_moe_combine(const MoeRowsParams& p, bool, int, hipStream_t) {
  printf("combine tokens=%ld rows=%ld X=%lu pos=%lu weights=%lu Y=%lu\n", (long)p.tokens, (long)p.rows, v(p.X), v(p.pos), v(p.weights), v(p.Y));
  return hipSuccess;
}
hipError_t launch_moe_combine_grad(const MoeRowsParams& p, bool, int, hipStream_t) {
  printf("grad tokens=%ld rows=%ld t0=%ld t1=%ld r0=%ld r1=%ld X=%lu Y=%lu\n", (long)p.tokens, (long)p.rows, (long)p.first_token,
         (long)p.end_token, (long)p.first_row, (long)p.end_row, v(p.X), v(p.Y));
  return hipSuccess;
}
}  // namespace sfc
int main() {
  char cmd[16];
  char *A = (char*)(1ul << 50), *B = (char*)(2ul << 50), *C = (char*)(3ul << 50), *D = (char*)(4ul << 50), *E = (char*)(5ul << 50);
  long a, b, c, d;
  while (scanf("%15s %ld %ld %ld %ld", cmd, &a, &b, &c, &d) == 5) {
    int rc = 1;
    auto q = [](long n) { return (n + 31) / 32 * 16; };
    auto z = [](long n) { return ((n + 31) / 32 + 3) / 4 * 4; };
    if (!strcmp(cmd, "quant"))        // rows cols outputs(1 rows 2 columns 3 both) topk(0: no order)
      rc = sfc_mx4_quant(a, b, A, b, 1, d ? (int*)E : nullptr, 77, (int)d, c & 1 ? B : nullptr, q(b), c & 1 ? C : nullptr, z(b),
                         c & 2 ? D : nullptr, q(a), c & 2 ? D + (1l << 49) : nullptr, z(a), nullptr);
    else if (!strcmp(cmd, "dequant")) rc = sfc_mx4_dequant(a, b, A, q(b), B, z(b), C, b, (int)c, nullptr);
    else if (!strcmp(cmd, "dispatch")) rc = sfc_moe_dispatch(a, b, 100, (int)c, A, b, (int)d, (int*)B, (float*)E, C, b, nullptr);
    else if (!strcmp(cmd, "combine")) rc = sfc_moe_combine(a, b, 1000, (int)c, A, b, (int)d, (int*)B, (float*)E, C, b, nullptr);
    else if (!strcmp(cmd, "grad"))
      rc = sfc_moe_combine_grad(a, b, c, (int)d, A, b, A, b, 0, (int*)B, (int*)B, (float*)E, C, b, (float*)D, nullptr);
    else if (!strcmp(cmd, "gemm")) rc = sfc_gemm_mx4_ex(a, b, c, A, q(c), B, z(c), C, q(c), D, z(c), E, b, (int)d, nullptr);
    printf("ret rc=%d\n", rc);
  }
  return 0;
}
'''
A, B, C, D, E = (i << 50 for i in range(1, 6))
THREADS = 1 << 32


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("ops_launches"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    main, out = os.path.join(d, "main.cpp"), os.path.join(d, "ops_launches")
    with open(main, "w") as f:
        f.write(host_api.MAIN.split("int main()")[0] + STUBS)
    src = [f"{host_api.CSRC}/{n}" for n in ("sfcgemm_api.cpp", "sfc_model.cpp", "sfc_ops_api.cpp")]
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", f"-I{d}", f"-I{host_api.ROOT}/include", f"-I{host_api.CSRC}", main,
                    *src, "-o", out], check=True)

    def run(*line):
        events, = host_api.run(out, [" ".join(str(x) for x in line)])
        assert events[-1] == ("ret", {"rc": 0})
        return events[:-1]
    return run


LONG = [1, 1000, 1 << 23, (1 << 23) + 1, (1 << 28) + 5, (1 << 31) - 1]
up = lambda v, m: -(-v // m) * m
codes = lambda n: up(n, 32) // 2
scales = lambda n: up(up(n, 32) // 32, 4)


@pytest.mark.parametrize("rows", LONG)
@pytest.mark.parametrize("cols", [1, 4097])
@pytest.mark.parametrize("topk", [0, 3])
def test_quant_along_rows(call, rows, cols, topk):
    first = 0
    for name, e in call("quant", rows, cols, 1, topk):
        assert name == "quant" and e["rows"] * 256 < THREADS and e["cols"] == cols
        assert e["X"] == A + (0 if topk else first * cols * 2) and e["order"] == (E + first * 4 if topk else 0)
        assert e["x_rows"] == (77 if topk else e["rows"])
        assert e["Q"] == B + first * codes(cols) and e["S"] == C + first * scales(cols) and e["Qt"] == e["St"] == 0
        first += e["rows"]
    assert first == rows


# (rows of codes lie less than 2^22 bytes apart: below 2^23 values along each axis that has blocks)
@pytest.mark.parametrize("rows,cols,axis", [(1, 1, 2), (1, 1, 3), (8192, 4096, 3), (5003, 2049, 2), (200, 1 << 20, 3), (1, (1 << 31) - 1, 2),
                                            (257, (1 << 28) + 77, 2), ((1 << 23) - 32, 100, 2), ((1 << 23) - 99, 8192 * 20 + 1, 3),
                                            ((1 << 22) + 5, (1 << 22) + 1, 3)])
@pytest.mark.parametrize("topk", [0, 2])
def test_quant_along_columns(call, rows, cols, axis, topk):
    events = call("quant", rows, cols, axis, topk)
    first = col = 0
    for name, e in events:
        assert name == "quant" and -(-e["rows"] // 128) * -(-e["cols"] // 128) * 512 < THREADS
        assert first % 256 == 0 and col % 128 == 0
        assert e["X"] == A + ((0 if topk else first * cols) + col) * 2 and e["order"] == (E + first * 4 if topk else 0)
        assert e["Qt"] == D + col * codes(rows) + first // 2
        assert e["St"] == D + (1 << 49) + col * scales(rows) + first // 32
        assert e["Q"] == (B + first * codes(cols) + col // 2 if axis == 3 else 0)
        assert e["S"] == (C + first * scales(cols) + col // 32 if axis == 3 else 0)
        col += e["cols"]
        if col == cols:
            first, col = first + e["rows"], 0
    assert first == rows and col == 0
    if -(-rows // 128) * -(-cols // 128) < 1 << 20:
        assert len(events) == 1


@pytest.mark.parametrize("rows", LONG)
@pytest.mark.parametrize("out", [0, 1])
def test_dequant(call, rows, out):
    first = 0
    for name, e in call("dequant", rows, 100, out, 0):
        assert e["rows"] * 256 < THREADS
        assert e["Q"] == A + first * codes(100) and e["S"] == B + first * scales(100) and e["Y"] == C + first * 100 * (2 if out else 4)
        first += e["rows"]
    assert first == rows


@pytest.mark.parametrize("rows", LONG)
@pytest.mark.parametrize("kind", [0, 1])
def test_dispatch(call, rows, kind):
    first = 0
    for name, e in call("dispatch", rows, 3, 2, kind):
        assert e["rows"] * 256 < THREADS and e["tokens"] == 100 and e["X"] == A and e["weights"] == E
        assert e["order"] == B + first * 4 and e["Y"] == C + first * 3 * (2 if kind else 4)
        first += e["rows"]
    assert first == rows


@pytest.mark.parametrize("tokens", LONG[:-1])
@pytest.mark.parametrize("kind", [0, 1])
def test_combine(call, tokens, kind):
    first = 0
    for name, e in call("combine", tokens, 3, 2, kind):
        assert e["tokens"] * 256 < THREADS and e["rows"] == 1000 and e["X"] == A
        assert e["pos"] == B + first * 8 and e["weights"] == E + first * 8 and e["Y"] == C + first * 3 * (2 if kind else 4)
        first += e["tokens"]
    assert first == tokens


@pytest.mark.parametrize("tokens,rows", [(1, 1), (8191, 17000), (0, 31), (31, 0), (1 << 23, 1 << 26), ((1 << 23) + 1, 5), (5, (1 << 28) + 1),
                                         (1 << 28, (1 << 31) - 1), ((1 << 31) - 1, 7)])
def test_gradient_of_combine(call, tokens, rows):
    t = r = 0
    events = call("grad", tokens, 3, rows, 1)
    for name, e in events:
        assert e["tokens"] == tokens and e["rows"] == rows and e["X"] == A and e["Y"] == C
        assert e["t0"] == t and e["r0"] == r
        t, r = e["t1"], e["r1"]
        assert ((t - e["t0"]) + -(-(r - e["r0"]) // 16)) * 256 < THREADS and (t > e["t0"] or r > e["r0"])
    assert t == tokens and r == rows
    if tokens <= 1 << 23 and rows <= 1 << 26:
        assert len(events) == 1


@pytest.mark.parametrize("N", [4096, (1 << 28) - 1, 1 << 28, (1 << 31) - 1])
def test_streaming_product(call, N):
    """512 threads take 32 columns; past 2^28 columns the products go to the block kernel, whose grid is bounded."""
    names = [n for n, _ in call("gemm", 20, N, 32, 1) if n in ("rows", "tile")]
    assert names == (["rows"] if N < 1 << 28 else ["tile"])
    if names == ["rows"]:
        assert -(-N // 32) * 512 <= THREADS - 512 or N == (1 << 28) - 1
