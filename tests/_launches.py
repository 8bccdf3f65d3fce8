"""What the library holds and would launch, without a GPU: in a process of its own the library is loaded behind stand-ins for the
few functions of the HIP runtime that it calls, which write down each kernel's name, grid, block and first arguments
and run nothing."""
import json
import os
import re
import subprocess
import sys

from paper_2606_07574_amd import build

STANDIN = r"""
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
typedef struct { uint32_t x, y, z; } dim3;
static struct { const void* f; const char* name; } known[4096];
static int count;
void** __hipRegisterFatBinary(const void* data) { static void* handle; (void)data; return &handle; }
void __hipUnregisterFatBinary(void** handle) { (void)handle; }
void __hipRegisterFunction(void** m, const void* f, char* device, const char* name, unsigned limit, void* tid, void* bid,
                           void* block, void* grid, int* size) {
    (void)m, (void)device, (void)limit, (void)tid, (void)bid, (void)block, (void)grid, (void)size;
    if (count < 4096) known[count].f = f, known[count++].name = name;
    printf("kernel %s\n", name);
    fflush(stdout);
}
int hipStreamGetDevice(void* stream, int* device) { (void)stream; *device = 0; return 0; }
int hipDeviceGetAttribute(int* value, int attribute, int device) { (void)attribute, (void)device; *value = 256; return 0; }
int hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, void* stream) {
    (void)lds, (void)stream;
    const char* name = "?";
    for (int k = 0; k < count; ++k)
        if (known[k].f == f) name = known[k].name;
    printf("launch %s %u %u %u %u %llu %d\n", name, grid.x, grid.y, grid.z, block.x,
           (unsigned long long)*(uint64_t*)args[0], *(int*)args[1]);
    fflush(stdout);
    return 0;
}
"""

DRIVER = r"""
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
kinds = {"p": ctypes.c_void_p, "i": ctypes.c_int, "l": ctypes.c_int64, "f": ctypes.c_float}
for line in sys.stdin:
    name, kind, args = json.loads(line)
    fn = getattr(lib, name)
    fn.argtypes = [ctypes.POINTER(ctypes.c_float) if k == "c" else kinds[k] for k in kind]
    fn.restype = ctypes.c_int64 if name.endswith("_work") else ctypes.c_int
    args = [(ctypes.c_float * len(a))(*a) if k == "c" else a for k, a in zip(kind, args)]
    print("done", fn(*args), flush=True)
"""


def split(name):
    """(kernel, its template's numbers) of a mangled name."""
    kernel, values = re.match(r"_ZN12_GLOBAL__N_1\d+([a-z_0-9]+?_kernel)(?:I((?:L[bi]\d+E)+)E)?", name).groups()
    return kernel, tuple(int(v) for v in re.findall(r"L[bi](\d+)E", values or ""))


def run(calls, folder):
    source, stub = os.path.join(folder, "standin.c"), os.path.join(folder, "libstandin.so")
    with open(source, "w") as f:
        f.write(STANDIN)
    subprocess.check_call(["gcc", "-O1", "-fPIC", "-shared", "-o", stub, source])
    run = subprocess.run([sys.executable, "-c", DRIVER, stub, build.LIB], input="\n".join(json.dumps(c) for c in calls), text=True,
                         capture_output=True, timeout=300)
    assert run.returncode == 0, run.stderr
    return [line.split() for line in run.stdout.splitlines()]


def kernels(folder):
    """All kernels of the library."""
    return {split(words[1]) for words in run([], folder) if words[0] == "kernel"}


def launches(calls, folder):
    """calls: (function, kinds of its arguments: p(ointer), i(nt), l(ong), f(loat), c(oefficients), arguments). For each
    (its code, [(kernel, its template's numbers, grid x, grid y, block, first argument, second one as an int)])."""
    found, now = [], []
    for word, *rest in run(calls, folder):
        if word == "done":
            found.append((int(rest[0]), now))
            now = []
        elif word == "launch":
            name, gx, gy, _, block, first, second = rest
            now.append((*split(name), int(gx), int(gy), int(block), int(first), int(second)))
    assert len(found) == len(calls)
    return found
