"""Which kernels, grids and memory a call of the experts' bf16 products or of the low-rank adapters takes: the host layer
run against the stand-in for the HIP runtime of host_api.py, so no GPU is needed."""
import os
import subprocess

import pytest

import host_api
from rows_cases import DEPTHS, EXPERTS, FEW
from test_ops_routes import STUBS as OPS_STUBS

STUBS = r'''
#include "sfc_moe_params.h"
#include "sfc_lora_params.h"
namespace sfc {
static hipError_t moe(int b, const MoeGemmParams& p, MoeLayout l, bool ob, int grid) {
  printf("tile b=%d layout=%d bf16=%d grid=%d gm=%d gn=%d M=%ld N=%ld table=%lu past=%d topk=%d\n", b, (int)l, (int)ob, grid, p.gm, p.gn,
         (long)p.M, (long)p.N, v(p.table), (int)p.past, p.topk);
  return hipSuccess;
}
hipError_t launch_moe_256x256(const MoeGemmParams& p, MoeLayout l, bool ob, int g, hipStream_t) { return moe(256, p, l, ob, g); }
hipError_t launch_moe_128x128(const MoeGemmParams& p, MoeLayout l, bool ob, int g, hipStream_t) { return moe(128, p, l, ob, g); }
hipError_t launch_moe_64x64(const MoeGemmParams& p, MoeLayout l, bool ob, int g, hipStream_t) { return moe(64, p, l, ob, g); }
hipError_t launch_moe_rows(const MoeGemmParams& p, int fm, int fn, bool ob, hipStream_t) {
  printf("rows fm=%d fn=%d bf16=%d experts=%d N=%ld\n", fm, fn, (int)ob, p.experts, (long)p.N);
  return hipSuccess;
}
static void lora(const char* name, const LoraParams& p, bool nk, bool bf16) {
  printf("%s rows=%ld cols=%ld nk=%d bf16=%d splits=%d ids=%lu X=%lu W=%lu V=%lu base=%lu Y=%lu sums=%lu parts=%lu byrows=%d\n", name, (long)p.rows,
         (long)p.cols, (int)nk, (int)bf16, p.splits, v(p.ids), v(p.X), v(p.W), v(p.V), v(p.base), v(p.Y), v(p.sums), v(p.parts),
         (int)lora_by_rows(p.rows, p.cols, p.rank));
}
hipError_t launch_lora_down(const LoraParams& p, bool nk, hipStream_t) { lora("down", p, nk, false); return hipSuccess; }
hipError_t launch_lora_up(const LoraParams& p, bool nk, bool bf16, int, hipStream_t) { lora("up", p, nk, bf16); return hipSuccess; }
hipError_t launch_lora_wgrad(const LoraParams& p, bool nk, bool bf16, hipStream_t) { lora("wgrad", p, nk, bf16); return hipSuccess; }
}  // namespace sfc
int main() {
  char cmd[16];
  long rows, n, k, groups, layout, type, pad;
  unsigned long s, ws, wb;
  void *A = (void*)(1ul << 50), *B = (void*)(2ul << 50), *C = (void*)(3ul << 50), *V = (void*)(4ul << 50), *I = (void*)(5ul << 50);
  while (scanf("%15s", cmd) == 1) {
    int rc = 0;
    if (!strcmp(cmd, "capture")) {
      if (scanf("%lu %ld", &s, &n) != 2) return 1;
      if (n) capturing.insert((hipStream_t)s);
      else capturing.erase((hipStream_t)s);
    } else {
      if (scanf("%ld %ld %ld %ld %ld %ld %ld %lu %lu %lu", &rows, &n, &k, &groups, &layout, &type, &pad, &ws, &wb, &s) != 10) return 1;
      const int E = (int)groups, lay = (int)layout, ty = (int)type;
      const long lb = (lay ? n : k) + pad, sb = (lay ? k : n) * lb;
      if (!strcmp(cmd, "experts")) rc = sfc_moe_gemm_ex(rows, n, k, E, A, k + pad, nullptr, 0, 0, B, lb, sb, lay, (int*)I, C, n, ty, (void*)s);
      else if (!strcmp(cmd, "depth")) rc = sfc_moe_wgrad_ex(n, k, rows, E, A, n + pad, B, k + pad, (int*)I, C, k, n * k, ty, (void*)s);
      // (adapters: n columns, k ranks)
      else if (!strcmp(cmd, "down")) rc = sfc_lora_down(rows, n, k, E, A, n, B, lay ? k : n, n * k, lay, (int*)I, nullptr, (float*)V, k, (void*)ws, wb, (void*)s);
      else if (!strcmp(cmd, "up")) rc = sfc_lora_up(rows, n, k, E, (float*)V, k, B, lay ? n : k, n * k, lay, (int*)I, A, n, C, n, ty, (void*)s);
      else if (!strcmp(cmd, "wgrad")) rc = sfc_lora_wgrad(rows, n, k, E, A, n, (float*)V, k, (int*)I, C, lay ? n : k, n * k, lay, ty, (void*)ws, wb, (void*)s);
      else if (!strcmp(cmd, "sizes")) printf("sizes down=%zu wgrad=%zu\n", sfc_lora_down_ws_size(rows, n, k, E), sfc_lora_wgrad_ws_size(rows, n, k, E));
      else return 1;
    }
    printf("ret rc=%d\n", rc);
  }
  return 0;
}
'''
A, B, C, V, I = (i << 50 for i in range(1, 6))


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("rows_routes"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    main, out = os.path.join(d, "main.cpp"), os.path.join(d, "rows_routes")
    with open(main, "w") as f:
        f.write(host_api.MAIN.split("int main()")[0] + OPS_STUBS.split("int main()")[0] + STUBS)
    src = [f"{host_api.CSRC}/{n}" for n in ("sfcgemm_api.cpp", "sfc_model.cpp", "sfc_ops_api.cpp", "sfc_rows_api.cpp")]
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", f"-I{d}", f"-I{host_api.ROOT}/include", f"-I{host_api.CSRC}", main, *src, "-o", out],
                   check=True)
    return out


def line(cmd, rows, n, k, groups, layout=0, out=0, pad=0, ws=0, ws_bytes=0, stream=1):
    return f"{cmd} {rows} {n} {k} {groups} {layout} {out} {pad} {ws} {ws_bytes} {stream}"


def one(exe, *a, **kw):
    events, = host_api.run(exe, [line(*a, **kw)])
    return events


def launches(events):
    assert events[-1] == ("ret", {"rc": 0})
    return [e for e in events if e[0] in ("tile", "rows", "down", "up", "wgrad")]


def kernel(exe, *a, **kw):
    (name, e), = launches(one(exe, *a, **kw))
    return f"rows{e['fm']}" if name == "rows" else str(e["b"])


# ---- experts -------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows,N,K,experts,nk,kn", [
    (2, 4096, 4096, 8, "rows1", "64"), (64, 4096, 4096, 8, "rows1", "128"), (512, 2048, 4096, 64, "rows1", "128"),
    (2, 4096, 4095, 8, "rows1", "64"), (32, 4096, 4095, 8, "128", "128"), (24, 4096, 4096, 1, "rows2", "64"), (64, 4096, 4096, 1, "rows4", "64"),
    (128, 4096, 4096, 8, "128", "128"), (1024, 4096, 4096, 8, "128", "128"), (4096, 14336, 4096, 8, "256", "256"),
    (16384, 4096, 4096, 8, "256", "256"), (1, 1, 1, 1, "64", "64"), (1, 1, 8, 1, "rows1", "64")])
def test_experts_kernel(exe, rows, N, K, experts, nk, kn):
    assert kernel(exe, "experts", rows, N, K, experts, 0) == nk and kernel(exe, "experts", rows, N, K, experts, 1) == kn


def test_the_gpu_tests_reach_every_kernel(exe):
    """What the shapes of rows_cases.py run on, and how their last rounds of blocks are taken."""
    got, ends, deep_ends = set(), set(), set()

    def end(b, total, grid):
        left = total % grid
        return b, total > grid, "none" if not left else "quarters" if b > 64 and 2 * left <= grid else "blocks"

    for c, N, K in EXPERTS:
        for layout in (0, 1):
            for pad in (0, 3):
                if not sum(c):
                    continue
                (name, e), = launches(one(exe, "experts", sum(c), N, K, len(c), layout, pad=pad))
                got.add((f"rows{e['fm']}" if name == "rows" else str(e["b"]), layout))
                if name == "tile":
                    ends.add(end(e["b"], sum(-(-n // e["b"]) for n in c) * e["gn"], e["grid"]))
    assert {(k, layout) for k in ("64", "128", "256") for layout in (0, 1)} | {("rows1", 0)} <= got
    assert {(128, True, "quarters"), (256, True, "quarters"), (64, False, "blocks"), (256, True, "blocks"), (128, True, "none")} <= ends
    assert {kernel(exe, "experts", sum(c) + 1, N, K, len(c)) for c, N, K in FEW} >= {"rows1", "rows2", "rows4"}
    for c, M, N in DEPTHS:
        (_, e), = launches(one(exe, "depth", sum(c), M, N, len(c)))
        deep_ends.add(end(e["b"], e["gm"] * e["gn"] * len(c), e["grid"]))
    assert {(64, False, "none"), (128, True, "quarters"), (256, True, "quarters"), (256, False, "none")} <= deep_ends


def past(elements, ld, depth, out):
    """Whether a result goes past the caches: 32 MB and more; 256 and more in whole 16-byte pieces of rows or behind a long depth."""
    size = 4 - 2 * out
    return elements * size >= 32 << 20 and (ld * size % 16 == 0 or -(-depth // 64) > 16 or elements * size < 256 << 20)


@pytest.mark.parametrize("out", [0, 1])
@pytest.mark.parametrize("rows,N,K,experts", [(5000, 4097, 1024, 8), (33000, 4097, 1024, 8), (33000, 4097, 1025, 8), (1000, 1407, 2047, 60), (1, 5, 9, 1), (300, 700, 64, 1024), (5000, 4100, 512, 8), (1 << 20, 14336, 4096, 8)])
def test_experts_grid(exe, rows, N, K, experts, out):
    for layout in (0, 1):
        (name, e), = launches(one(exe, "experts", rows, N, K, experts, layout, out))
        if name == "tile":
            assert e["layout"] == layout and e["bf16"] == out and e["gn"] == -(-N // e["b"]) and e["past"] == past(rows * N, N, K, out)
            assert 1 <= e["grid"] <= 256 * {256: 1, 128: 2, 64: 4}[e["b"]]
    (_, e), = launches(one(exe, "depth", rows, N, K, experts, 0, out))
    assert e["layout"] == 2 and e["table"] and e["gm"] == -(-N // e["b"]) and e["gn"] == -(-K // e["b"])
    assert 1 <= e["grid"] <= min(e["gm"] * e["gn"] * experts, 1024) and e["past"] == past(N * K * experts, K, -(-rows // experts), out)


def test_experts_without_work_take_no_launch(exe):
    for a in (("experts", 0, 8, 8, 2), ("experts", 8, 0, 8, 2), ("depth", 8, 0, 8, 2), ("depth", 8, 8, 0, 2)):
        assert launches(one(exe, *a)) == []
    assert len(launches(one(exe, "experts", 8, 8, 0, 2))) == len(launches(one(exe, "depth", 0, 8, 8, 2))) == 1          # zeros


# ---- adapters ------------------------------------------------------------------------------------


@pytest.mark.parametrize("rows,n,rank,by_rows", [(1, 4096, 16, 1), (64, 14336, 64, 1), (256, 14336, 16, 1), (256, 14336, 64, 0),
                                                 (512, 4096, 16, 1), (2048, 4096, 64, 0), (4096, 4096, 64, 0), (4097, 8, 1, 0), (4096, 8, 1, 1)])
def test_rows_one_by_one(exe, rows, n, rank, by_rows):
    for cmd in ("down", "up"):
        (_, e), = launches(one(exe, cmd, rows, n, rank, 4))
        assert e["byrows"] == by_rows


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rows,cols", [((1 << 21) + 5, 16), ((1 << 22) + 1, 4096), ((1 << 18) + 3, (1 << 20) + 9), (70000, 3 << 20)])
def test_long_batches_are_cut_without_a_gap(exe, rows, cols, layout):
    rank = 16
    events = launches(one(exe, "up", rows, cols, rank, 2, layout, 1))
    seen = 0
    for _, e in events:
        first, col = (e["ids"] - I) // 4, (e["Y"] - C) // 2 % cols
        assert e["Y"] == C + 2 * (first * cols + col) and e["base"] == A + 2 * (first * cols + col) and e["V"] == V + 4 * first * rank
        assert e["W"] == B + 2 * (col if layout else col * rank)
        assert first + e["rows"] <= rows and col + e["cols"] <= cols
        # 256 threads for 64 columns and 256 rows where that makes 512 workgroups, else for 64 rows
        wide = -(-e["cols"] // 64)
        assert max(wide * -(-e["rows"] // 256), min(wide * -(-e["rows"] // 64), 2048)) * 256 < 1 << 32
        seen += e["rows"] * e["cols"]
    assert seen == rows * cols and len({(e["ids"], e["Y"]) for _, e in events}) == len(events) > 1
    if cols < 1 << 20:
        parts = launches(one(exe, "down", rows, cols, rank, 2, layout))
        at = 0
        for _, e in parts:
            assert e["ids"] == I + 4 * at and e["X"] == A + 2 * at * cols and e["V"] == V + 4 * at * rank
            at += e["rows"]
        assert at == rows


@pytest.mark.parametrize("rows,n,rank,adapters", [(4096, 4096, 64, 8), (8192, 4096, 16, 16), (2001, 2040, 24, 5), (300, 4096, 16, 3), (20, 64, 8, 2),
                                                  (8192, 4096, 16, 1), (100000, 512, 256, 1025), ((1 << 21) + 5000, 4096, 64, 2)])
def test_workspaces(exe, rows, n, rank, adapters):
    sizes = dict(one(exe, "sizes", rows, n, rank, adapters))["sizes"]
    for cmd in ("down", "wgrad"):
        need = sizes[cmd]
        events = one(exe, cmd, rows, n, rank, adapters)
        assert ("malloc" in dict(events) or "malloc_async" in dict(events)) == (need > 0)
        if not need:
            assert all(e["sums"] == 0 for _, e in launches(events))
            continue
        ws = 1 << 40
        with_ws = one(exe, cmd, rows, n, rank, adapters, ws=ws, ws_bytes=need)
        assert not {"malloc", "malloc_async"} & set(dict(with_ws))
        for _, e in launches(with_ws):
            if e["splits"] > 1:
                table = (8 * adapters + 15) // 16 * 16 if cmd == "wgrad" else 0
                size = e["splits"] * rank * (e["rows"] if cmd == "down" else n) * 4
                assert e["sums"] == ws + table and table + size <= need and (cmd == "down" or e["parts"] == ws)
        short, = host_api.run(exe, [line(cmd, rows, n, rank, adapters, ws=ws, ws_bytes=need - 1)])
        assert launches_none(short) and short[-1][1]["rc"] == -3
        again = one(exe, cmd, rows, n, rank, adapters, ws=ws, ws_bytes=0)
        assert again[-1][1]["rc"] == -3


def launches_none(events):
    return not [e for e in events if e[0] in ("down", "wgrad")]


@pytest.mark.parametrize("cmd", ["down", "wgrad"])
def test_memory_of_graphs(exe, cmd):
    """Recorded calls have library memory of their own, of the stream they are recorded on."""
    f = lambda s: line(cmd, 4096, 4096, 64, 8, stream=s)  # noqa: E731
    eager, _, rec, _, again, other = host_api.run(exe, [f(1), "capture 1 1", f(1), "capture 1 0", f(1), f(2)])
    at = [dict(e)[cmd]["sums"] for e in (eager, rec, again, other)]
    assert all(at) and at[0] == at[2] and len({at[0], at[1], at[3]}) == 3


def test_most_adapters_with_parts(exe):
    """More adapters than are counted in one workgroup take no parts."""
    (_, few), = launches(one(exe, "wgrad", 100000, 512, 16, 1024))
    (_, many), = launches(one(exe, "wgrad", 100000, 512, 16, 1025))
    assert few["splits"] > 1 and many["splits"] == 1
