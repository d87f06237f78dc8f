"""What the library launches for a call, without a GPU: the calls run in a process of their own whose HIP launches and function
attributes go to a recorder in place of the runtime (test infrastructure; nothing is launched, no pointer is read)."""
from __future__ import annotations

import ctypes
import json
import os
import subprocess
import sys
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RECORDER = r"""
#include <cxxabi.h>
#include <dlfcn.h>
#include <cstddef>
#include <cstdio>
#include <cstdlib>
struct dim3 { unsigned x, y, z; };
static FILE* out;
static struct { dim3 grid, block; size_t lds; void* stream; } pushed;
static void write(const char* kind, const void* f, long long a, long long b, long long c) {
    Dl_info i;
    const char* n = dladdr(f, &i) && i.dli_sname ? i.dli_sname : "?";
    int st;
    char* d = abi::__cxa_demangle(n, nullptr, nullptr, &st);
    fprintf(out, "%s|%s|%lld|%lld|%lld\n", kind, d ? d : n, a, b, c);
    free(d);
}
extern "C" {
void recorder_open(const char* path) { out = fopen(path, "w"); }
void recorder_close() { fclose(out); }
void recorder_call(int status) { fprintf(out, "call|%d\n", status); }
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, void* s) { pushed = {g, b, lds, s}; return 0; }
int __hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, void** s) { *g = pushed.grid; *b = pushed.block; *lds = pushed.lds; *s = pushed.stream; return 0; }
int hipLaunchKernel(const void* f, dim3 g, dim3 b, void**, size_t lds, void*) { write("launch", f, g.x, b.x, static_cast<long long>(lds)); return 0; }
int hipFuncSetAttribute(const void* f, int what, int value) { write("attribute", f, what, value, 0); return 0; }
int hipGetLastError() { return 0; }
}
"""


def record(calls):
    """calls: [entry, sizes ...] as in _run below.  For each: its status, launches [(kernel, workgroups, threads, bytes of LDS)] and function
    attributes [(kernel, attribute, value)]."""
    with tempfile.TemporaryDirectory() as d:
        src, lib, log = (os.path.join(d, n) for n in ("recorder.cpp", "recorder.so", "log"))
        with open(src, "w") as f:
            f.write(RECORDER)
        subprocess.run(["g++", "-O1", "-shared", "-fPIC", src, "-o", lib, "-ldl"], check=True)
        env = dict(os.environ, PYTHONPATH=ROOT, HIP_VISIBLE_DEVICES="-1")
        subprocess.run([sys.executable, os.path.abspath(__file__), lib, log, json.dumps(calls)], check=True, env=env, timeout=300)
        with open(log) as f:
            lines = [l.rstrip("\n").split("|") for l in f]
    out, launches, attributes = [], [], []
    for l in lines:
        if l[0] == "call":
            out.append({"status": int(l[1]), "launches": launches, "attributes": attributes})
            launches, attributes = [], []
            continue
        name = l[1].replace("void ", "").replace("loka::", "").split("(")[0]
        if l[0] == "launch":
            launches.append((name, int(l[2]), int(l[3]), int(l[4])))
        else:
            attributes.append((name, int(l[2]), int(l[3])))
    assert len(out) == len(calls)
    return out


def _run(L, B, call):
    p, ref, room = ctypes.c_void_p(0x1000), ctypes.byref, 1 << 60
    name, *a = call
    if name == "route":                # tokens, experts, top_k, bf16
        T, E, k, bf16 = a
        return L.loka_route(ref(B.RouteDesc(T, E, E, k, B.SCORE_SOFTMAX, 1, int(bf16), 1.0)), p, p, p, p, p, p, p, room, None)
    if name == "quantize":             # rows, cols, groups, x_rows (0: no index), along, turned
        rows, cols, groups, x_rows, along, turned = a
        q, t = (p if along else None), (p if turned else None)
        return L.loka_grouped_quantize(ref(B.GroupedQuantizeDesc(rows, cols, cols, x_rows, groups)), p, p if x_rows else None, p, q, q, t, t, None)
    rows, N, K, groups = a[:4]
    d = B.GroupedDesc(rows, rows, N, K, groups, B.W_TURNED if len(a) < 5 or a[4] else B.W_ALONG)
    if name == "gemm":                 # rows, N, K, groups, weights turned
        return L.loka_grouped_gemm(ref(d), p, p, None, p, p, p, p, None, None)
    if name == "linear":
        return L.loka_grouped_linear(ref(d), p, K, None, p, p, p, p, None, p, room, None)
    assert name == "wgrad"
    return L.loka_grouped_wgrad(ref(d), p, p, p, p, p, p, None, p, room, None)


def _main():
    rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)             # ahead of the runtime, so that the library finds these first
    from paper_2605_10886_amd import binding as B

    L = B.lib()
    for name in ("hipLaunchKernel", "hipFuncSetAttribute", "hipGetLastError", "__hipPushCallConfiguration", "__hipPopCallConfiguration"):
        a, b = (ctypes.cast(getattr(l, name), ctypes.c_void_p).value for l in (rec, ctypes.CDLL(None)))
        assert a == b, name
    rec.recorder_open(sys.argv[2].encode())
    for call in json.loads(sys.argv[3]):
        rec.recorder_call(_run(L, B, call))
    rec.recorder_close()


if __name__ == "__main__":
    _main()
