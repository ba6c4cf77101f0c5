"""Every kernel of the low-rank adapters that the library holds is taken by a shape of the GPU tests, and the shapes with infinities and
NaN are taken in tiles: the rules of sfc_lora_params.h, compiled with g++, against the compiler's notes.  No GPU is needed."""
import os
import subprocess

import pytest

import host_api
import kernel_notes
from lora_cases import SPECIAL, TALL
from test_gpu_lora import SHAPES

MAIN = r'''
#include <hip/hip_runtime.h>
#include <stdio.h>
#include "sfc_lora_params.h"
int main() {
  long rows, cols;
  int rank, adapters;
  while (scanf("%ld %ld %d %d", &rows, &cols, &rank, &adapters) == 4)
    printf("%d %d %d %d %d %d %d %d %d %d %d\n", (int)sfc::lora_by_rows(rows, cols, rank), sfc::lora_row_ranks(rows, rank),
           sfc::lora_row_lanes(rank, 32), sfc::lora_row_lanes(rank, 8), sfc::lora_up_chunks(rank), sfc::lora_up_tiles(rows, cols, rank, false, 256),
           sfc::lora_up_tiles(rows, cols, rank, true, 256), sfc::lora_down_splits(rows, cols, rank, 256), (int)sfc::lora_grad_narrow(cols, rank),
           sfc::lora_grad_ranks(cols, rank), sfc::lora_wgrad_splits(rows, cols, rank, adapters, 256));
  return 0;
}
'''


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("lora_rules"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    main, exe = os.path.join(d, "main.cpp"), os.path.join(d, "rules")
    with open(main, "w") as f:
        f.write(MAIN)
    subprocess.run(["g++", "-std=c++17", "-w", f"-I{d}", f"-I{host_api.CSRC}", main, "-o", exe], check=True)
    names = ("by_rows", "ranks", "lanes32", "lanes8", "chunks", "tiles_f32", "tiles_bf16", "down_splits", "narrow", "grad_ranks", "grad_splits")

    def ask(shapes):
        text = "".join("%d %d %d %d\n" % s for s in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [dict(zip(names, map(int, line.split()))) for line in out.splitlines()]
    return ask


def cpp(*values):
    return "<" + ", ".join(str(v).lower() for v in values) + ">"


def up(r):
    """Kernels of up for both layouts and types."""
    for bf16 in (False, True):
        if r["by_rows"]:
            yield "lora_row_up_kn" + cpp(bf16)
            yield "lora_row_up_nk" + cpp(r["lanes8"], bf16)
        else:
            for nk in (False, True):
                yield "lora_up_kernel" + cpp(r["tiles_bf16" if bf16 else "tiles_f32"], r["chunks"], nk, bf16)


def down(r, rank):
    if r["by_rows"]:
        yield "lora_row_down_nk" + cpp(r["ranks"])
        yield "lora_row_down_kn" + cpp(r["lanes32"])
    else:
        yield from ("lora_down_kernel<true>", "lora_down_kernel<false>")
        if r["down_splits"] > 1:
            yield "lora_down_sum" + cpp(16 if rank <= 16 else 64)


def gradient(r):
    for bf16 in (False, True):
        for nk in (False, True):
            yield "lora_wgrad_kernel" + cpp(r["grad_ranks"], bool(r["narrow"]), nk, bf16)
        if r["grad_splits"] > 1:
            yield "lora_grad_sum" + cpp(bf16)


def test_every_kernel_is_taken_by_a_gpu_test(rules):
    taken = set()
    for shape, r in zip(SHAPES, rules(SHAPES)):
        taken |= {*up(r), *down(r, shape[2]), *gradient(r)}
    for r in rules(TALL):
        taken |= {*up(r)}
    compiled = {n for n in kernel_notes.kernels() if n.startswith("lora_")}
    assert taken == compiled


def test_tall_shapes_have_256_rows_to_a_workgroup(rules):
    for r in rules(TALL):
        assert not r["by_rows"] and r["tiles_f32"] == r["tiles_bf16"] == 4
    assert {r["chunks"] for r in rules(TALL)} == {1, 2, 4, 8}


def test_special_values_are_met_in_tiles(rules):
    """Infinities and NaN: every chunk count of up, every form of the gradient."""
    got = rules(SPECIAL)
    assert not any(r["by_rows"] for r in got)
    assert {r["chunks"] for r in got} == {1, 2, 4, 8} and {r["narrow"] for r in got} == {0, 1}
    assert {r["grad_splits"] > 1 for r in got} == {False, True}
