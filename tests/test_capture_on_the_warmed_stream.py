"""Calls recorded on the stream that made their curve table: HIP refuses to ask after an event that was last recorded on a stream
that is being captured, and ends the capture.  The stand-in for the HIP runtime of host_api.py with that rule, and with words of
host memory that the device writes.  No GPU is needed."""
import os
import subprocess

import pytest

import host_api
from host_api import gemm

# events know the stream they were last recorded on; fills of host words take place once the device is ready
RULE = r'''
#include <map>
#include <vector>
static std::map<hipEvent_t, hipStream_t> recorded;
static int32_t host_words[64];
static int words_used = 0;
static std::vector<int32_t*> pending;
'''


def replaced(text, old, new):
    assert text.count(old) == 1
    return text.replace(old, new)


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d = str(tmp_path_factory.mktemp("warmed"))
    os.makedirs(os.path.join(d, "hip"))
    with open(os.path.join(d, "hip", "hip_runtime.h"), "w") as f:
        f.write(host_api.HIP)
    main = replaced(host_api.MAIN, "static int fail_in = 0, not_ready = 0;", "static int fail_in = 0, not_ready = 0;" + RULE)
    main = replaced(main, "hipError_t hipEventQuery(hipEvent_t) {", "hipError_t hipEventQuery(hipEvent_t ev) {\n  if (capturing.count(recorded[ev])) { printf(\"ended_capture a=1\\n\"); return (hipError_t)907; }")
    main = replaced(main, "{ *e = (hipEvent_t)8; return hipSuccess; }", "{ static uintptr_t n = 8; *e = (hipEvent_t)n++; return hipSuccess; }")
    main = replaced(main, "hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }",
                    "hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) { recorded[e] = s; return hipSuccess; }")
    main = replaced(main, "hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t, unsigned) {",
                    "hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t e, unsigned) {\n"
                    "  if (capturing.count(recorded[e])) printf(\"joined_capture a=1\\n\");\n  else printf(\"waited stream=%lu\\n\", (unsigned long)(uintptr_t)s);")
    main = replaced(main, "hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }",
                    "hipError_t hipGetDevice(int* d) {\n  if (!not_ready) { for (int32_t* p : pending) *p = 1; pending.clear(); }\n  *d = 0;\n  return hipSuccess;\n}")
    main = replaced(main, "  printf(\"fill p=%lu n=%ld\\n\", u(p), (long)n);",
                    "  if (p >= host_words && p < host_words + 64) { pending.push_back(p); return hipSuccess; }\n  printf(\"fill p=%lu n=%ld\\n\", u(p), (long)n);")
    main = replaced(main, "hipError_t run_mfma_probe", "volatile int32_t* host_word() { return host_words + words_used++; }\nhipError_t run_mfma_probe")
    with open(os.path.join(d, "main.cpp"), "w") as f:
        f.write(main)
    out = os.path.join(d, "warmed")
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", f"-I{d}", f"-I{host_api.ROOT}/include", f"-I{host_api.CSRC}", os.path.join(d, "main.cpp"),
                    f"{host_api.CSRC}/sfcgemm_api.cpp", f"{host_api.CSRC}/sfc_model.cpp", "-o", out], check=True)
    return out


CALLS = [dict(M=900, N=1300, K=600, tile=3), dict(M=4000, N=14000, K=1000), dict(M=16, N=12520, K=7656, ca=0)]


def tables(events):
    return [e["table"] for n, e in events if n == "gemm"]


def orders(events):
    return [e["d"] for n, e in events if n == "order"]


def fine(calls):
    for c in calls:
        assert c[-1] == ("ret", {"rc": 0})
        assert not {"ended_capture", "joined_capture"} & {n for n, _ in c}


@pytest.mark.parametrize("a", CALLS)
def test_a_table_that_is_ready(exe, a):
    """One call, the device done with it, then the recording: the table is used as it is."""
    call = gemm("ex", **a, stream=1)
    calls = host_api.run(exe, ["notready 1", call, "notready 0", "capture 1 1", call, call, "capture 1 0", call])
    fine(calls)
    for i in (4, 5, 7):
        assert tables(calls[i]) == tables(calls[1]) == orders(calls[1]) and not orders(calls[i])


@pytest.mark.parametrize("a", CALLS)
def test_a_table_that_may_not_be_ready(exe, a):
    """The recorded call writes a table of its own; one that runs at once on another stream waits, or where the table's stream
    is being captured makes its own."""
    one, two = gemm("ex", **a, stream=1), gemm("ex", **a, stream=2)
    calls = host_api.run(exe, ["notready 1", one, two, "capture 1 1", one, two, "capture 1 0", one, "notready 0", two])
    fine(calls)
    first, waits, recorded, beside, same, last = (calls[i] for i in (1, 2, 4, 5, 7, 9))
    assert tables(waits) == tables(first) and not orders(waits) and "waited" in dict(waits)
    assert tables(recorded) == orders(recorded) and not set(tables(recorded)) & set(tables(first))
    if orders(beside):
        assert tables(beside) == orders(beside)
    assert "waited" not in dict(beside) and not set(tables(beside)) & set(tables(first) + tables(recorded))
    assert tables(same) == tables(last) == tables(beside)
